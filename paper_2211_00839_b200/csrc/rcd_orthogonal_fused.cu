// All steps of rcd_orthogonalize in one launch, for matrices whose products take less time than the launches between them.
//
// One CTA per SM, resident together (a cooperative launch).  A step is three phases: A = X X^T, B = b A + c A A, X = a X + B X (or their mirrored forms for a
// tall X); a barrier over the grid lies between two phases.  Within a phase a CTA takes tiles of 128 x 64: operands by TMA in boxes of 64 x 64, which serve either order and either side;
// one thread issues tcgen05.mma; eight warps finish a tile from tensor memory, a lane a row of 32 columns.  Where a phase has few tiles and a long k axis, a team of two or four CTAs
// of a cluster shares a tile: each pushes its sums of the others' rows into their shared memory and finishes its own rows, adding in the order of the pieces.
//
// 512 x 2048 takes 111 us where fifteen launches take 155: a phase 5 to 7, of which the barrier takes 1.6 (the stores' way, one report per CTA, the others' look at
// the count), the first slab's way 0.9, a slab 0.3 to 0.36 (24 KB from L2 for every SM at once), a tile in pieces 1.8.  What bounds it is this chain, not the rate of anything.
//
// The roles go through the phases by themselves: the warp that loads waits for the count and tells those that finish; a warp of its own reports.  Every wait is
// bounded; whoever waits in vain leaves, and the others behind it.
#include "rcd_orthogonal.h"
#include "rcd_tc.cuh"
#include "rcd_walk.h"

namespace rcd {

namespace {

constexpr int kRows = 128, kCols = 64, kBoxBytes = 64 * 128, kStage = 3 * kBoxBytes, kStages = 7, kThreads = 384, kFirstFinisher = 4, kFinishers = 8;
constexpr int kMostTeam = 4;                                           // CTAs that share a tile; a cluster is a team of the phase with the largest
constexpr int kPartial = kRows * kCols * 4;
constexpr uint32_t kWaitTurns = 1u << 16, kPolls = 1u << 21;           // about a second either

struct __align__(8) FusedShared {
    uint64_t full[kStages], empty[kStages], accFull[2], accEmpty[2];
    uint64_t open;                         // the phase before is complete on all SMs
    uint64_t done;                         // this phase is on this one
    uint64_t partials;                     // the team's sums of this CTA's rows are here
    uint32_t tmemBase;
    int32_t abort;
    Unit units[3][kFusedUnits];            // what this CTA does in the phases of a step
    int32_t count[3];
};
constexpr int kSharedBytes = kStages * kStage + kPartial + (int)sizeof(FusedShared);

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
// The grid's barrier: a count of CTAs that have finished a phase.
__device__ __forceinline__ void count_in(uint32_t *counter) { asm volatile("red.release.gpu.global.add.u32 [%0], 1;" :: "l"(counter) : "memory"); }
__device__ __forceinline__ bool wait_for_count(const uint32_t *counter, uint32_t target, FusedShared *sh, uint32_t polls = kPolls)
{
    for (uint32_t poll = 0; poll < polls; ++poll) {
        uint32_t v;
        asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
        if ((int32_t)(v - target) >= 0) {
            __threadfence();                                           // (what was written before the others' reports)
            return true;
        }
        if (*(volatile int32_t *)&sh->abort) return false;
    }
    atomicExch(&sh->abort, 1);
    return false;
}
// The address of the same variable in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t team_addr(const void *p, int rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    return a;
}
// Four numbers to another CTA's shared memory, reported to its barrier when they are there.
__device__ __forceinline__ void push(uint32_t to, uint32_t bar, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%2, %3, %4, %5}, [%1];" :: "r"(to), "r"(bar), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// The same descriptor as make_smem_desc for an operand whose k elements lie next to each other; for the other order boxes of 64 x 64 follow one another.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool across)
{
    const uint64_t d = make_smem_desc(addr);
    return across ? (d & ~((uint64_t)0x3fff << 16)) | (uint64_t)(kBoxBytes >> 4) << 16 : d;
}

__global__ void __launch_bounds__(kThreads, 1)
newton_schulz_kernel(const __grid_constant__ CUtensorMap mapX0, const __grid_constant__ CUtensorMap mapX1, const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                     const __grid_constant__ FusedParams p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    float *const partial = reinterpret_cast<float *>(smem + kStages * kStage);
    FusedShared &sh = *reinterpret_cast<FusedShared *>(smem + kStages * kStage + kPartial);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = (int)blockIdx.x & (p.cluster - 1);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh.accFull[b], 1); mbar_init(&sh.accEmpty[b], kFinishers); }
        mbar_init(&sh.partials, 1);
        mbar_init(&sh.open, 1);
        mbar_init(&sh.done, kFinishers);
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_addr(&sh.tmemBase)), "r"(2 * kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 2 && lane < 3) {
        // the tiles of this CTA, of each kind of phase (a tile in pieces: a team's)
        const FusedPhase &f = p.phases[lane];
        const Walk w{f.tiles / f.tilesN, f.tilesN, f.tiles, f.tilesN, 1, f.symmetric ? 1 : 0, f.symmetric ? 2 : 0};
        const int tiles = f.tiles * p.batch, first = (int)blockIdx.x / f.team, step = (int)gridDim.x / f.team;
        int n = 0;
        for (int u = first; u < tiles && n < kFusedUnits; u += step) {
            Unit t = unit_of(w, u % f.tiles);
            t.batch = u / f.tiles;
            sh.units[lane][n++] = t;
        }
        sh.count[lane] = n;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                     // the team's barriers exist
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmemBase = sh.tmemBase;
    const int phases = 3 * p.steps;
    const float down = 1.0f / (1 << kUp);

    // Every role goes through the phases by itself; where it has waited in vain it leaves, and the others behind it.
    if (warp == 0) {
        // ---------------- operands; and whether the phase before is complete ----------------
        const bool leader = elect_one();
        int s = 0;
        uint32_t parity = 1;
        bool ok = true;
        for (int ph = 0, kind = 0, odd = 0; ph < phases && ok; ++ph) {
            const FusedPhase &f = p.phases[kind];
            const CUtensorMap *const mapX = odd ? &mapX1 : &mapX0;
            const CUtensorMap *const a = kind == 0 ? mapX : kind == 1 ? &mapA : p.tall ? mapX : &mapB;
            const CUtensorMap *const b = kind == 0 ? mapX : kind == 1 ? &mapA : p.tall ? &mapB : mapX;
            const int begin = rank % f.team * f.per, end = min(f.slabs, begin + f.per), count = sh.count[kind];
            if (ph > 0) {
                if (!__all_sync(0xffffffffu, wait_for_count(p.counter, (uint32_t)ph * gridDim.x, &sh))) break;
                proxy_fence();                                         // (what was written there by ordinary stores is read by TMA from here on)
                if (leader) mbar_arrive(&sh.open);
            }
            for (int n = 0; n < count && ok; ++n) {
                const Unit t = sh.units[kind][n];
                const int m0 = t.m * kRows, n0 = t.n * kCols, aRow = t.batch * f.stepA, bRow = t.batch * f.stepB;
                for (int kb = begin; kb < end; ++kb) {
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
            if (++kind == 3) { kind = 0; odd ^= 1; }
        }
    } else if (warp == 1) {
        // ---------------- products ----------------
        const bool leader = elect_one();
        int s = 0;
        uint32_t parity = 0, nt = 0;
        bool ok = true;
        for (int ph = 0, kind = 0; ph < phases && ok; ++ph) {
            const FusedPhase &f = p.phases[kind];
            const uint32_t idesc = (1u << 4) | (f.acrossA ? 1u << 15 : 0u) | (f.acrossB ? 1u << 16 : 0u) | ((uint32_t)(kCols >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
            const uint64_t stepA = f.acrossA ? 128 : 2, stepB = f.acrossB ? 128 : 2;
            const int begin = rank % f.team * f.per, end = min(f.slabs, begin + f.per), count = sh.count[kind];
            for (int n = 0; n < count && ok; ++n, ++nt) {
                const uint32_t buf = nt & 1;
                if (!warp_wait_for(&sh.accEmpty[buf], ((nt >> 1) & 1) ^ 1, &sh)) { ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
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
            if (++kind == 3) kind = 0;
        }
    } else if (warp == 2) {
        // ---------------- one report per CTA and phase (eight, from every warp that finishes, queue up at the counter: 2 us with 128 CTAs) ----------------
        for (int ph = 0; ph + 1 < phases; ++ph) {
            if (!warp_wait_for(&sh.done, ph & 1, &sh)) break;
            if (lane == 0) count_in(p.counter);
        }
    } else if (warp >= kFirstFinisher) {
        // ---------------- finish: quarter q of the rows, half of the columns ----------------
        const int q = warp & 3, half = (warp - kFirstFinisher) >> 2, me = (int)threadIdx.x - 32 * kFirstFinisher;
        uint32_t nt = 0, shares = 0;
        bool ok = true;
        for (int ph = 0, kind = 0, odd = 0; ph < phases && ok; ++ph) {
            const FusedPhase &f = p.phases[kind];
            const bool last = ph == phases - 1, residualWanted = kind > 0;
            const float *const c = p.coefficients + ph - kind;
            const float alpha0 = kind == 0 ? down : kind == 1 ? c[2] * down : last ? down * down : down, beta0 = kind == 1 ? c[1] : last ? c[0] * down : c[0];
            const int64_t square = (int64_t)p.side * p.side, whole = (int64_t)p.rows * p.cols;
            const int count = sh.count[kind];
            if (ph > 0 && !warp_wait_for(&sh.open, (ph - 1) & 1, &sh)) break;
            for (int n = 0; n < count && ok; ++n, ++nt) {
                const Unit t = sh.units[kind][n];
                const uint32_t buf = nt & 1;
                const float factor = ph < 3 && kind != 1 ? p.factor[t.batch] : 1.0f;        // (of the first step: G is brought up by a power of two alone)
                const float alpha = kind == 0 ? alpha0 * (factor * factor) : alpha0 * factor, beta = beta0 * factor;
                const int row0 = t.m * kRows, col0 = t.n * kCols;
                const __half *const from = kind == 1 ? p.a + t.batch * square : (odd ? p.x1 : p.x0) + t.batch * whole;      // residual: [M][N]
                __half *const to = kind == 0 ? p.a + t.batch * square : kind == 1 ? p.b + t.batch * square : (odd ? p.x0 : p.x1) + t.batch * whole;
                auto residual_of = [&](int row, int col) { return __ldcg(reinterpret_cast<const uint4 *>(from + (int64_t)row * f.N + col)); };
                // eight neighbours of a row, from fp32 sums on
                auto put = [&](int row, int col, float (&z)[8], const uint4 &r) {
                    const int64_t at = (int64_t)row * f.N + col;
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] *= alpha;
                    if (residualWanted) {
                        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
                            z[2 * j] = fmaf(beta, v.x, z[2 * j]);
                            z[2 * j + 1] = fmaf(beta, v.y, z[2 * j + 1]);
                        }
                        if (ph == 2 && p.low) {
                            float l[8];
                            load_pack<8>(l, p.low + t.batch * whole + at);
#pragma unroll
                            for (int j = 0; j < 8; ++j) z[j] = fmaf(beta * (1.0f / (1 << kLowUp)), l[j], z[j]);
                        }
                    }
                    if (last) {
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
                if (residualWanted && f.team == 1 && inside) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) residual[k] = residual_of(row, col0 + half * 32 + 8 * k);
                }
                if (!warp_wait_for(&sh.accFull[buf], (nt >> 1) & 1, &sh)) { ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t v[32];
                tmem_load_32cols(tmemBase + buf * kCols + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * 32), v);
                tmem_load_wait();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.accEmpty[buf]);
                if (f.team == 1) {
                    if (inside) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float z[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(v[8 * k + j]);
                            put(row, col0 + half * 32 + 8 * k, z, residual[k]);
                        }
                    }
                } else {
                    // Each of the team finishes its share of the rows, whole quarters: all send it their pieces' sums of them (16 bytes at a time, turned by the row: no bank
                    // twice).  One tile per team and phase: a phase has ended on all SMs between two uses of the place.
                    if (me == 0) mbar_expect_tx(&sh.partials, kPartial);
                    const int team = f.team, share = kRows / team, member = rank % team, source = kPartial / 4 / team;       // source: floats that come from one of the team
                    const int owner = rank - member + q * team / 4, at = (q % (4 / team)) * 32 + lane;
                    const uint32_t to = team_addr(partial + member * source + at * kCols, owner), bar = team_addr(&sh.partials, owner);
#pragma unroll
                    for (int k = 0; k < 8; ++k) push(to + (((half * 8 + k) ^ (lane & 15)) << 4), bar, v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                    if (!warp_wait_for(&sh.partials, shares & 1, &sh)) { ok = false; break; }
                    ++shares;
                    const int col = me % (kCols / 8) * 8;              // 256 threads: 32 rows of 8 times 8 columns at a time
                    for (int r = me / (kCols / 8); r < share; r += 32) {
                        const int mine = row0 + member * share + r;
                        if (mine >= f.M || col0 >= f.N) break;
                        const uint4 old = residualWanted ? residual_of(mine, col0 + col) : uint4{};
                        float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                        for (int k = 0; k < team; ++k) {
                            const float *const from = partial + k * source + r * kCols;
                            const float4 lo = *reinterpret_cast<const float4 *>(from + (((col / 4) ^ (r & 15)) << 2)), hi = *reinterpret_cast<const float4 *>(from + (((col / 4 + 1) ^ (r & 15)) << 2));
                            z[0] += lo.x; z[1] += lo.y; z[2] += lo.z; z[3] += lo.w;
                            z[4] += hi.x; z[5] += hi.y; z[6] += hi.z; z[7] += hi.w;
                        }
                        put(mine, col0 + col, z, old);
                    }
                }
            }
            if (!ok || last) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.done);
            if (++kind == 3) { kind = 0; odd ^= 1; }
        }
    }
    if (*(volatile int32_t *)&sh.abort) let_copies_land();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                     // nobody reads this CTA's place any more
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmemBase), "r"(2 * kCols) : "memory");
    }
    if (threadIdx.x == 0 && sh.abort) atomicOr(p.status, kDevTimeout);
}

// The waits of all steps in one launch for a count that nobody reaches and for an arrival that nobody makes: the first has to run out for every thread, and the one
// behind it to be given up at once.
__global__ void __launch_bounds__(64) fused_wait_selftest_kernel(uint32_t *counter, int32_t *status)
{
    __shared__ FusedShared sh;
    if (threadIdx.x == 0) {
        sh.abort = 0;
        mbar_init(&sh.open, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const bool came = wait_for_count(counter, *(volatile uint32_t *)counter + 1, &sh, 1u << 10);
    const bool then = wait_for(&sh.open, 0, &sh);
    const bool wrong = __syncthreads_or(came || then);
    if (threadIdx.x == 0) atomicOr(status, wrong || !sh.abort ? kDevBadState : kDevTimeout);
}

}  // namespace

rcd_status launch_fused_wait_selftest(rcd_ctx *ctx, int32_t *status, cudaStream_t st)
{
    fused_wait_selftest_kernel<<<1, 64, 0, st>>>((uint32_t *)ctx->statusOwn + kSelftestCount, status);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

static cudaLaunchConfig_t fused_launch(int64_t grid, int cluster, cudaLaunchAttribute (&attrs)[2])
{
    attrs[0].id = cudaLaunchAttributeCooperative;
    attrs[0].val.cooperative = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = (unsigned)cluster;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)grid);
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = kSharedBytes;
    config.attrs = attrs;
    config.numAttrs = cluster > 1 ? 2 : 1;                // (a profiler may not take both: ncu 2025 does not)
    return config;
}

// CTAs in clusters of 1, 2 and 4 that the device takes at once (some of its groups of SMs are not whole fours: 148, 148 and 132 of 148).
static int ctas_of(rcd_ctx *ctx, int log2Cluster)
{
    int &known = ctx->fusedCtas[log2Cluster];
    if (known < 0) {
        known = 0;
        if (!ctx->cooperative || cudaSetDevice(ctx->device) != cudaSuccess || allow_shared(newton_schulz_kernel, kSharedBytes) != cudaSuccess) return 0;
        const int cluster = 1 << log2Cluster;
        cudaLaunchAttribute attrs[2];
        const cudaLaunchConfig_t config = fused_launch(ctx->smCount / cluster * cluster, cluster, attrs);
        int n = 0;
        if (cluster == 1) known = ctx->smCount;            // (one of them fills an SM's shared memory)
        else if (cudaOccupancyMaxActiveClusters(&n, newton_schulz_kernel, &config) == cudaSuccess) known = std::min(n * cluster, ctx->smCount);
        else cudaGetLastError();
    }
    return known;
}

FusedPlan fused_plan(rcd_ctx *ctx, int64_t batch, int64_t rows, int64_t cols, bool tall)
{
    FusedPlan best{};
    const int64_t side = std::min(rows, cols), sideTiles = (side + kRows - 1) / kRows;
    if (side > 4096 || rows > (1 << 20) || cols > (1 << 20)) return best;
    for (int log2Cluster = 0; (1 << log2Cluster) <= kMostTeam; ++log2Cluster) {
        FusedPlan f{};
        f.cluster = 1 << log2Cluster;
        const int64_t ctas = ctas_of(ctx, log2Cluster);
        int64_t most = 0;
        bool fits = ctas > 0;
        for (int k = 0; k < 3 && fits; ++k) {
            FusedPhase &ph = f.phases[k];
            ph.symmetric = k < 2;
            ph.M = (int32_t)(k < 2 ? side : rows);
            ph.N = (int32_t)(k < 2 ? side : cols);
            ph.slabs = (int32_t)((k == 0 ? std::max(rows, cols) : side) / 64);
            ph.acrossA = k == 0 && tall;
            ph.acrossB = k == 0 ? tall : k == 2 && !tall;
            ph.stepA = (int32_t)(k == 0 ? rows : k == 1 ? side : tall ? rows : side);
            ph.stepB = (int32_t)(k == 0 ? rows : k == 1 ? side : tall ? side : rows);
            ph.tilesN = (int32_t)(ph.N / kCols);
            const int64_t tiles = k < 2 ? sideTiles * (sideTiles + 1) : (rows + kRows - 1) / kRows * (cols / kCols);
            fits = tiles * batch <= ctas * kFusedUnits;
            ph.tiles = (int32_t)tiles;
            // A phase takes 2.7 us besides its slabs of 0.36 each (the barrier over the grid 1.6, the first slab's way and the last tile's end); a tile in pieces 1.8 more.
            double least = 1e300;
            for (int team = 1; team <= f.cluster; team *= 2) {
                const int64_t per = (ph.slabs + team - 1) / team;
                if (team > 1 && (tiles * batch * team > ctas || (team - 1) * per >= ph.slabs)) continue;       // (a tile for every team, and no empty piece)
                const double t = 2.7 + (double)((tiles * batch * team + ctas - 1) / ctas) * 0.36 * (double)per + (team > 1 ? 1.8 : 0.0);
                if (t < least) {
                    least = t;
                    ph.team = team;
                    ph.per = (int32_t)per;
                }
            }
            f.stepUs += least;
            most = std::max(most, tiles * batch * ph.team);
        }
        if (!fits || (best.possible && f.stepUs >= best.stepUs)) continue;
        f.grid = (int32_t)(std::min<int64_t>((most + f.cluster - 1) / f.cluster, ctas / f.cluster) * f.cluster);
        f.possible = true;
        best = f;
    }
    return best;
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
    void *args[5] = {&maps[0], &maps[1], &maps[2], &maps[3], const_cast<FusedParams *>(&p)};
    cudaLaunchAttribute attrs[2];
    cudaLaunchConfig_t config = fused_launch(plan.grid, plan.cluster, attrs);
    config.stream = st;
    ctx->kernelLaunches++;
    ctx->tcLaunches++;
    RCD_CUDA(ctx, cudaLaunchKernelExC(&config, (const void *)newton_schulz_kernel, args));
    return RCD_OK;
}

}  // namespace rcd

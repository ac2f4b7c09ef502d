// Matrix products of rcd_linear and its gradients on the tensor cores:  C = A B^T with an epilogue, or C as partial sums of a
// piece of the k axis, which a second kernel joins.
//
// Persistent CTAs (one per SM), or pairs of CTAs on one tile (cta_group::2: each holds half of A's rows and half of B's, so an
// operand row comes in once for 256 rows of the other).  Operand tiles come by TMA in slabs of 128 bytes of k (64 elements of
// 16 bits, 128 of 8) with the 128-byte swizzle into a ring; an operand whose m or n elements lie next to each other instead of its k
// elements (`across`: the gradients' transposed factors) comes in boxes of 64 such elements by 64 k and is multiplied as it lies
// (the instruction takes either order).  One thread issues tcgen05.mma into one of two 256-column accumulators in tensor
// memory, so that eight warps finish a tile while the next one is computed: 32 columns at a time from tensor memory, times the scales,
// plus bias, activation, plus residual, rounded into 32 rows x 128 bytes of shared memory, and out by TMA.  The residual's piece
// comes in by TMA into the same place one piece ahead.  Rows that a tensor map cannot describe (they do not start on 16 bytes)
// are first copied (operands), or moved between that place and memory by the warp itself (outputs, residual); so are the ends of output
// rows that do not end on 16 bytes: a TMA store writes the last 16 bytes that an element of the row lies in whole.
//
// Warp roles: 0 = TMA producer, 1 = TMEM allocation + MMA issue, 2..9 = epilogue, two per quarter of the TMEM lanes.
// Every wait is bounded, as in the similarity kernel: on expiry the CTA records kDevTimeout and leaves.
#include "rcd_act.cuh"
#include "rcd_linear.h"
#include "rcd_norm.cuh"
#include "rcd_tc.cuh"

namespace rcd {

namespace {

constexpr int kRows = 128;                              // rows of A per CTA
constexpr int kSlab = 128;                              // bytes of k per operand row and stage
constexpr int kSlabRows16 = 64;                         // k elements of 16 bits per slab
constexpr int kBox = 64 * kSlab;                        // 8 KB: 64 k rows of 64 elements
constexpr int kABytes = kRows * kSlab;
constexpr int kMostStages = 8;
constexpr int kEpiWarps = 8;
// The tensor cores cut an fp32 sum off where they cannot hold it, towards zero: products of fp16 and of one sign lose 6.5e-9 of the result
// each, 3.2e-4 over 50 000 (two thirds of the type's half step).  So sums are taken in chunks that are added up outside with rounding.
// fp32 outputs: 512 k (2.4e-6 within a chunk, bf16 2.3e-7, and half a unit of fp32 at most for each of them).  16-bit outputs: 2048 k (1.3e-5)
// where a piece has more than 4096, up to which the loss is a twentieth of fp16's half step.  (Gradients of 2048 x 2048 weights over 600 000
// rows: 3.56 ms in chunks, 3.45 in one sum.)
constexpr int kChunkSlabs = 8, kChunkSlabs16 = 32;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kPiece = 32 * 128;                        // an epilogue warp's piece of the output: 32 rows of 128 bytes
constexpr int kStaging = kEpiWarps * 2 * kPiece;
constexpr int kColumnBytes = kEpiWarps * 2 * 32 * 4;    // 32 biases and 32 scales per warp
constexpr uint32_t kWaitTurns = 1u << 16;               // of at most 20 us: a second or so
constexpr int kMostShared = 227 * 1024;

struct __align__(8) Shared {
    uint64_t full[kMostStages], empty[kMostStages];     // full: CTA 0's of a pair
    uint64_t accFull[2], accEmpty[2];                   // accEmpty: CTA 0's of a pair
    uint64_t residual[kEpiWarps][2];
    uint32_t tmemBase;
    int32_t abort;
};
constexpr int kFixedShared = kStaging + kColumnBytes + (int)sizeof(Shared);

struct TcParams {
    int32_t M, N, tilesN, tiles, units, slabs, slabsPerSplit, chunk, tn, stages, stageBytes, rowsPart;
    uint32_t idesc;
    Epilogue e;
    bool raw;                                           // accumulators as they are, into e.y: [split][rowsPart][ldy]
    bool tmaY, tmaZ, tmaR, edgeByHand;                  // edgeByHand: a piece that holds the rows' ends, since TMA stores 16 bytes at a time
    int32_t *status;
};

// (Suspended by the hardware up to 20 us at a time: polls with pauses cost the ring half a slab's time at every turn.)
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, Shared *sh, uint32_t turns = kWaitTurns)
{
    for (uint32_t turn = 0; turn < turns; ++turn) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity), "r"(20000) : "memory");
        if (ok) return true;
        if (*(volatile int32_t *)&sh->abort) return false;
    }
    atomicExch(&sh->abort, 1);
    return false;
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t mine;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(mine));
    return mine != 0;
}
// wait_for a whole warp, which goes on together or gives up together.
__device__ __forceinline__ bool warp_wait_for(uint64_t *bar, uint32_t parity, Shared *sh, uint32_t turns = kWaitTurns)
{
    return __all_sync(0xffffffffu, wait_for(bar, parity, sh, turns));
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, const void *src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                 :: "l"(map), "r"(smem_addr(src)), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" :: "n"(kLeft) : "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Descriptor of an operand whose m (n) elements lie next to each other: boxes of 64 of them (128 bytes) by 64 k, 8 KB apart; groups of 8 k
// are 1024 bytes apart.
__device__ __forceinline__ uint64_t across_desc(uint32_t addr)
{
    uint64_t d = make_smem_desc(addr) & ~((uint64_t)0x3fff << 16);
    return d | (uint64_t)(kBox >> 4) << 16;
}

// Byte of (row, 16-byte chunk) in a piece, as the 128-byte swizzle places it.
__device__ __forceinline__ int piece_at(int row, int chunk) { return row * 128 + ((chunk ^ (row & 7)) << 4); }

// A piece between its place in shared memory and rows that TMA cannot reach: element by element, neighbours by neighbouring lanes.
template <bool kLoad, typename T>
__device__ __forceinline__ void move_piece(unsigned char *piece, T *at, int64_t ld, int rows, int cols)
{
    constexpr int kCols = 128 / sizeof(T);
    const int lane = threadIdx.x & 31;
    rows = min(rows, 32);
    // (eight rows' accesses under way at once)
    for (int r0 = 0; r0 < rows; r0 += 8) {
        T v[8][kCols / 32];
        auto each = [&](auto go) {
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    const int row = r0 + r, col = c * 32 + lane;
                    if (row < rows && col < cols) go(v[r][c], *reinterpret_cast<T *>(piece + piece_at(row, col * (int)sizeof(T) / 16) + col * (int)sizeof(T) % 16), at[(int64_t)row * ld + col]);
                }
        };
        if constexpr (kLoad) {
            each([](T &x, T &, T &there) { x = there; });
            each([](T &x, T &here, T &) { here = x; });
        } else {
            each([](T &x, T &here, T &) { x = here; });
            each([](T &x, T &, T &there) { there = x; });
        }
    }
}

// 32 fp32 values to one row's 64 or 128 bytes of a piece, from 16-byte chunk `chunk` on.
__device__ __forceinline__ uint32_t pack2(float a, float b, rcd_elem type)
{
    if (type == RCD_ELEM_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 unpack2(uint32_t x, rcd_elem type)
{
    if (type == RCD_ELEM_BF16) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&x));
}
__device__ __forceinline__ void put_row(unsigned char *piece, int row, int chunk, const float (&v)[32], rcd_elem type)
{
    if (type == RCD_ELEM_F32) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            *reinterpret_cast<float4 *>(piece + piece_at(row, c)) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint4 *>(piece + piece_at(row, chunk + c)) =
                make_uint4(pack2(v[8 * c], v[8 * c + 1], type), pack2(v[8 * c + 2], v[8 * c + 3], type), pack2(v[8 * c + 4], v[8 * c + 5], type),
                           pack2(v[8 * c + 6], v[8 * c + 7], type));
    }
}
__device__ __forceinline__ void add_row(const unsigned char *piece, int row, int chunk, float (&v)[32], rcd_elem type)
{
    if (type == RCD_ELEM_F32) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float4 x = *reinterpret_cast<const float4 *>(piece + piece_at(row, c));
            v[4 * c] += x.x; v[4 * c + 1] += x.y; v[4 * c + 2] += x.z; v[4 * c + 3] += x.w;
        }
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint4 x = *reinterpret_cast<const uint4 *>(piece + piece_at(row, chunk + c));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2(w[i], type);
                v[8 * c + 2 * i] += f.x;
                v[8 * c + 2 * i + 1] += f.y;
            }
        }
    }
}
// Unit of work -> row tile, first column, piece of the k axis.  Column tiles are neighbours: the CTAs at work share a few row tiles of A
// and all of B.
struct Unit { int m, n, split; };
__device__ __forceinline__ Unit unit_of(const TcParams &p, int u)
{
    Unit t;
    t.split = u / p.tiles;
    u -= t.split * p.tiles;
    t.m = u / p.tilesN;
    t.n = (u - t.m * p.tilesN) * p.tn;
    return t;
}

// kChunks: 0, or the columns of a piece of the output, whose sums are taken in chunks.
template <bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks, bool kPair>
__device__ __forceinline__ void product_body(const CUtensorMap &mapA, const CUtensorMap &mapB, const CUtensorMap &mapY, const CUtensorMap &mapZ, const CUtensorMap &mapR, const TcParams &p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char *const tiles = smem;
    unsigned char *const staging = smem + (size_t)p.stages * p.stageBytes;
    float *const columns = reinterpret_cast<float *>(staging + kStaging);
    Shared &sh = *reinterpret_cast<Shared *>(staging + kStaging + kColumnBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kPair ? (int)(blockIdx.x & 1) : 0;
    const int first = kPair ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, step = kPair ? (int)(gridDim.x >> 1) : (int)gridDim.x;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMostStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh.accFull[b], 1); mbar_init(&sh.accEmpty[b], (kPair ? 2 : 1) * kEpiWarps); }
        for (int w = 0; w < kEpiWarps; ++w) { mbar_init(&sh.residual[w][0], 1); mbar_init(&sh.residual[w][1], 1); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (kPair) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_addr(&sh.tmemBase)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_addr(&sh.tmemBase)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (kPair) cluster_barrier();              // the other CTA's barriers exist
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmemBase = sh.tmemBase;
    const int rowsPerTile = kPair ? 2 * kRows : kRows;
    const int nMine = kPair ? p.tn / 2 : p.tn;           // B's rows that this CTA brings in

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        // (The whole warp goes through the loop, one lane issues: addresses stay in uniform registers, which is where these instructions
        // want them.  With the loop inside one lane's branch a slab took the issuer 600 cycles whatever its size.)
        const bool leader = elect_one();
        int s = 0;
        uint32_t phase = 1;
        bool ok = true;
        const int slabElems = kInt8 ? kSlab : kSlab / 2;
        const uint32_t bytes = (uint32_t)(kPair ? 2 : 1) * (uint32_t)(kABytes + nMine * kSlab);
        for (int u = first; u < p.units && ok; u += step) {
            const Unit t = unit_of(p, u);
            const int m0 = t.m * rowsPerTile + rank * kRows, n0 = t.n + rank * nMine;
            const int end = min(p.slabs, (t.split + 1) * p.slabsPerSplit);
            for (int kb = t.split * p.slabsPerSplit; kb < end; ++kb) {
                if (!warp_wait_for(&sh.empty[s], phase, &sh)) { ok = false; break; }
                unsigned char *a = tiles + s * p.stageBytes, *b = a + kABytes;
                if (leader) {
                    if (rank == 0) mbar_expect_tx(&sh.full[s], bytes);
                    uint32_t bar = smem_addr(&sh.full[s]);
                    if constexpr (kPair) bar = leader_addr(&sh.full[s]);
                    auto load = [&](void *dst, const CUtensorMap *map, int c0, int c1) {
                        if constexpr (kPair) pair_load_2d(dst, map, c0, c1, bar);
                        else tma_load_2d(dst, map, c0, c1, &sh.full[s]);
                    };
                    if constexpr (kAcrossA) {
#pragma unroll
                        for (int j = 0; j < kRows / 64; ++j) load(a + j * kBox, &mapA, m0 + 64 * j, kb * kSlabRows16);
                    } else {
                        load(a, &mapA, kb * slabElems, m0);
                    }
                    if constexpr (kAcrossB) {
                        for (int j = 0; j < nMine / 64; ++j) load(b + j * kBox, &mapB, n0 + 64 * j, kb * kSlabRows16);
                    } else {
                        load(b, &mapB, kb * slabElems, n0);
                    }
                }
                __syncwarp();
                if (++s == p.stages) { s = 0; phase ^= 1; }
            }
        }
        // after an abort: let the copies already issued land (a pair's report to CTA 0, so by time)
        if (*(volatile int32_t *)&sh.abort) let_copies_land();
    } else if (warp == 1) {
        // ---------------- MMA issuer (a pair's first CTA, for both) ----------------
        if (rank == 0) {
            const bool leader = elect_one();
            int s = 0;
            uint32_t phase = 0, nt = 0;
            bool ok = true;
            const uint32_t tile0 = smem_addr(tiles);
            for (int u = first; u < p.units && ok; u += step) {
                const Unit t = unit_of(p, u);
                const int end = min(p.slabs, (t.split + 1) * p.slabsPerSplit);
                for (int begin = t.split * p.slabsPerSplit; begin < end && ok; begin += p.chunk, ++nt) {
                    const uint32_t buf = nt & 1;
                    if (!warp_wait_for(&sh.accEmpty[buf], ((nt >> 1) & 1) ^ 1, &sh)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t tmemD = tmemBase + buf * 256;
                    const int stop = min(end, begin + p.chunk);
                    for (int kb = begin; kb < stop; ++kb) {
                        if (!warp_wait_for(&sh.full[s], phase, &sh)) { ok = false; break; }
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t aAddr = tile0 + (uint32_t)(s * p.stageBytes), bAddr = aAddr + kABytes;
                        const uint64_t descA = kAcrossA ? across_desc(aAddr) : make_smem_desc(aAddr);
                        const uint64_t descB = kAcrossB ? across_desc(bAddr) : make_smem_desc(bAddr);
                        // one MMA takes 32 bytes of k per row, or 16 rows of k of 128 bytes each
                        constexpr uint64_t kStepA = kAcrossA ? 128 : 2, kStepB = kAcrossB ? 128 : 2;
                        if (leader) {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if constexpr (kPair) pair_mma<kInt8>(tmemD, descA + kStepA * k, descB + kStepB * k, p.idesc, (kb > begin || k > 0) ? 1u : 0u);
                                else mma_issue<kInt8>(tmemD, descA + kStepA * k, descB + kStepB * k, p.idesc, (kb > begin || k > 0) ? 1u : 0u);
                            }
                            if constexpr (kPair) pair_commit(&sh.empty[s]);
                            else mma_commit(&sh.empty[s]);
                        }
                        __syncwarp();
                        if (++s == p.stages) { s = 0; phase ^= 1; }
                    }
                    if (leader) {
                        if constexpr (kPair) pair_commit(&sh.accFull[buf]);
                        else mma_commit(&sh.accFull[buf]);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        // ---------------- epilogue: this CTA's 128 rows ----------------
        const int q = warp & 3, ew = warp - 2, half = ew >> 2;       // TMEM lanes 32 q ..; pieces half, half + 2, ...
        unsigned char *const mine = staging + ew * 2 * kPiece;
        float *const biases = columns + ew * 64, *const scales = biases + 32;
        const Epilogue &e = p.e;
        const int wide = kChunks ? kChunks : e.type == RCD_ELEM_F32 ? 32 : 64;        // columns of a piece
        const int pieces = p.tn / wide;
        // a piece's coordinates; false where nothing of it lies inside the output
        struct Piece { int row, col; };
        auto piece_of = [&](int u, int k, Piece *o) {
            const Unit t = unit_of(p, u);
            o->row = t.m * rowsPerTile + rank * kRows + q * 32;
            o->col = t.n + k * wide;
            return o->row < p.M && o->col < p.N;
        };
        // the residual of the next piece that has one, from (u, k) on, is on its way into buffer `to`
        auto fetch = [&](int u, int k, int to) {
            Piece o;
            for (; u < p.units; u += step, k = half)
                for (; k < pieces; k += 2)
                    if (piece_of(u, k, &o)) {
                        mbar_expect_tx(&sh.residual[ew][to], kPiece);
                        tma_load_2d(mine + to * kPiece, &mapR, o.col, o.row, &sh.residual[ew][to]);
                        return;
                    }
        };
        const bool alternate = e.z == nullptr;                        // two buffers in turn, or one for y and one for z
        uint32_t nt = 0, turn = 0;
        if (p.tmaR && lane == 0) fetch(first, half, 0);
        bool ok = true;
        unsigned char *yPiece = mine;
        unsigned char *const zPiece = mine + kPiece;
        // a piece's place in shared memory is free, and the residual lies there
        auto begin_piece = [&](int u, int k, const Piece &o) {
            yPiece = mine + (alternate ? (turn & 1) * kPiece : 0);
            // (what was stored from it has been read out of it; a residual that comes next needs the other place too)
            if (lane == 0) {
                if (alternate && !p.tmaR) bulk_wait_read<1>();
                else bulk_wait_read<0>();
            }
            __syncwarp();
            if (p.tmaR) {
                if (alternate && lane == 0) fetch(u, k + 2, (turn & 1) ^ 1);
                // (with z in the other buffer the residual is fetched when the last piece has left)
                return warp_wait_for(&sh.residual[ew][alternate ? turn & 1 : 0], alternate ? (turn >> 1) & 1 : turn & 1, &sh);
            }
            if (e.residual) {
                if (e.type == RCD_ELEM_F32) move_piece<true>(yPiece, (float *)e.residual + (int64_t)o.row * e.ldr + o.col, e.ldr, p.M - o.row, p.N - o.col);
                else move_piece<true>(yPiece, (uint16_t *)e.residual + (int64_t)o.row * e.ldr + o.col, e.ldr, p.M - o.row, p.N - o.col);
                __syncwarp();
            }
            return true;
        };
        // The biases and scales of the warp's columns of a tile, 32 at a time (up to four times): asked for before the tile is ready, since
        // memory takes longer to answer than 32 columns take to finish; and those of one time to all lanes.
        const bool anyColumns = !p.raw && (e.bias || e.ws);
        float bias4[4], scale4[4];
        auto ask_columns = [&](const Unit &t) {
            if (!anyColumns) return;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int col = t.n + (wide == 64 ? (half + 2 * (c >> 1)) * 64 + (c & 1) * 32 : (half + 2 * c) * 32) + lane;
                bias4[c] = e.bias && col < p.N ? e.bias[col] : 0.0f;
                scale4[c] = e.ws && col < p.N ? e.ws[col] : 1.0f;
            }
        };
        auto columns_of = [&](int c) {
            if (!anyColumns) return;
            __syncwarp();
            biases[lane] = c == 0 ? bias4[0] : c == 1 ? bias4[1] : c == 2 ? bias4[2] : bias4[3];
            scales[lane] = c == 0 ? scale4[0] : c == 1 ? scale4[1] : c == 2 ? scale4[2] : scale4[3];
            __syncwarp();
        };
        // 32 columns of the lane's row, from column h of the piece on
        auto finish = [&](float (&z)[32], float sx, int h) {
            if (!p.raw) {
                if constexpr (kInt8) {
                    if (e.xs) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] *= sx;
                    }
                    if (e.ws) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 w = reinterpret_cast<const float4 *>(scales)[j / 4];
                            z[j] *= w.x; z[j + 1] *= w.y; z[j + 2] *= w.z; z[j + 3] *= w.w;
                        }
                    }
                }
                if (e.bias) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 b = reinterpret_cast<const float4 *>(biases)[j / 4];
                        z[j] += b.x; z[j + 1] += b.y; z[j + 2] += b.z; z[j + 3] += b.w;
                    }
                }
                if (e.z) put_row(zPiece, lane, h / 8, z, e.type);
                activate(z, e.act);
                if (e.residual) add_row(yPiece, lane, h / 8, z, e.type);
            }
            put_row(yPiece, lane, h / 8, z, e.type);
        };
        auto end_piece = [&](int u, int k, const Piece &o, int rowBase) {
            // (for the stores that leave from here by TMA, and for the next residual that TMA writes here: either comes after these ordinary writes)
            if (p.tmaY || p.tmaZ || p.tmaR) proxy_fence();
            __syncwarp();
            auto send = [&](bool byTma, const CUtensorMap *map, unsigned char *piece, void *to, int64_t ld, int base) {
                if (byTma && !(p.edgeByHand && o.col + wide > p.N)) {
                    if (lane == 0) tma_store_2d(map, piece, o.col, base + o.row);
                } else if (e.type == RCD_ELEM_F32) {
                    move_piece<false>(piece, (float *)to + ((int64_t)base + o.row) * ld + o.col, ld, p.M - o.row, p.N - o.col);
                } else {
                    move_piece<false>(piece, (uint16_t *)to + ((int64_t)base + o.row) * ld + o.col, ld, p.M - o.row, p.N - o.col);
                }
            };
            send(p.tmaY, &mapY, yPiece, e.y, e.ldy, rowBase);
            if (e.z) send(p.tmaZ, &mapZ, zPiece, e.z, e.ldz, 0);
            if (lane == 0) bulk_commit();
            __syncwarp();
            if (p.tmaR && !alternate && lane == 0) {
                bulk_wait_read<0>();
                fetch(u, k + 2, 0);
            }
            ++turn;
        };
        // hands an accumulator back
        auto release = [&](uint32_t buf) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if constexpr (kPair) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(leader_addr(&sh.accEmpty[buf])) : "memory");
                else mbar_arrive(&sh.accEmpty[buf]);
            }
        };
        for (int u = first; u < p.units && ok; u += step) {
            const Unit t = unit_of(p, u);
            const int rowBase = p.raw ? t.split * p.rowsPart : 0;
            const int row = t.m * rowsPerTile + rank * kRows + q * 32 + lane;
            const float sx = kInt8 && e.xs && row < p.M ? e.xs[row] : 1.0f;
            const uint32_t lanes = (uint32_t)(q * 32) << 16;
            ask_columns(t);
            if constexpr (kChunks != 0) {
                // Sums of chunks (see kChunkSlabs) in a lane's 128 registers, four times 32 columns; the next chunk is computed meanwhile.
                float sum[4][32];
                const int end = min(p.slabs, (t.split + 1) * p.slabsPerSplit);
                for (int begin = t.split * p.slabsPerSplit; begin < end && ok; begin += p.chunk, ++nt) {
                    const uint32_t buf = nt & 1;
                    if (!warp_wait_for(&sh.accFull[buf], (nt >> 1) & 1, &sh)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const bool fresh = begin == t.split * p.slabsPerSplit;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int col = wide == 64 ? (half + 2 * (i >> 1)) * 64 + (i & 1) * 32 : (half + 2 * i) * 32;
                        if (col < p.tn) {
                            uint32_t v[32];
                            tmem_load_32cols(tmemBase + buf * 256 + lanes + (uint32_t)col, v);
                            tmem_load_wait();
#pragma unroll
                            for (int j = 0; j < 32; ++j) sum[i][j] = fresh ? __uint_as_float(v[j]) : sum[i][j] + __uint_as_float(v[j]);
                        }
                    }
                    release(buf);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = wide == 64 ? half + 2 * (i >> 1) : half + 2 * i, h = wide == 64 ? (i & 1) * 32 : 0;
                    Piece o;
                    if (ok && k < pieces && piece_of(u, k, &o)) {
                        if (h == 0) ok = begin_piece(u, k, o);
                        if (ok) {
                            columns_of(i);
                            finish(sum[i], sx, h);
                            if (h + 32 == wide) end_piece(u, k, o, rowBase);
                        }
                    }
                }
            } else {
                const uint32_t buf = nt & 1;
                if (!warp_wait_for(&sh.accFull[buf], (nt >> 1) & 1, &sh)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int k = half; k < pieces; k += 2) {
                    Piece o;
                    if (!piece_of(u, k, &o)) continue;
                    if (!begin_piece(u, k, o)) { ok = false; break; }
                    for (int h = 0; h < wide; h += 32) {
                        uint32_t v[32];
                        tmem_load_32cols(tmemBase + buf * 256 + lanes + (uint32_t)(k * wide + h), v);
                        columns_of(wide == 64 ? (k - half) + h / 32 : (k - half) / 2);
                        tmem_load_wait();
                        float z[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = kInt8 && !p.raw ? (float)(int32_t)v[j] : __uint_as_float(v[j]);      // (raw integers stay what they are)
                        finish(z, sx, h);
                    }
                    end_piece(u, k, o, rowBase);
                }
                release(buf);
                ++nt;
            }
        }
        if (lane == 0) bulk_wait();
        if (!ok || *(volatile int32_t *)&sh.abort)                    // a residual may be on its way
            let_copies_land();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (kPair) cluster_barrier();              // nothing of the other CTA is on its way here any more
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if constexpr (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmemBase), "r"(512) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmemBase), "r"(512) : "memory");
    }
    if (threadIdx.x == 0 && sh.abort) atomicOr(p.status, kDevTimeout);
}

#define RCD_PRODUCT_ARGS const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapY, \
                         const __grid_constant__ CUtensorMap mapZ, const __grid_constant__ CUtensorMap mapR, const __grid_constant__ TcParams p
template <bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks = 0>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(RCD_PRODUCT_ARGS)
{
    product_body<kInt8, kAcrossA, kAcrossB, kChunks, false>(mapA, mapB, mapY, mapZ, mapR, p);
}
template <bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks = 0>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) product_pair_kernel(RCD_PRODUCT_ARGS)
{
    product_body<kInt8, kAcrossA, kAcrossB, kChunks, true>(mapA, mapB, mapY, mapZ, mapR, p);
}

// Joins the pieces of the k axis in their order, then the epilogue: four columns per thread.
template <bool kInt8>
__global__ void __launch_bounds__(256) join_kernel(const void *__restrict__ parts, int32_t splits, int32_t M, int64_t rowsPart, int32_t N, int64_t ld, const __grid_constant__ Epilogue e)
{
    const int perRow = (N + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)M * perRow) return;
    const int64_t m = i / perRow;
    const int n = (int)(i - m * perRow) * 4;
    float z[4];
    if constexpr (kInt8) {
        int4 s = make_int4(0, 0, 0, 0);
        for (int k = 0; k < splits; ++k) {
            const int4 x = __ldcs((const int4 *)((const int32_t *)parts + (k * rowsPart + m) * ld + n));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        z[0] = (float)s.x; z[1] = (float)s.y; z[2] = (float)s.z; z[3] = (float)s.w;
    } else {
        float4 s = make_float4(0, 0, 0, 0);
        for (int k = 0; k < splits; ++k) {
            const float4 x = __ldcs((const float4 *)((const float *)parts + (k * rowsPart + m) * ld + n));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        z[0] = s.x; z[1] = s.y; z[2] = s.z; z[3] = s.w;
    }
    const float sx = e.xs ? e.xs[m] : 1.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (n + j >= N) break;
        z[j] *= sx;
        if (e.ws) z[j] *= e.ws[n + j];
        if (e.bias) z[j] += e.bias[n + j];
    }
    const int64_t eb = e.type == RCD_ELEM_F32 ? 4 : 2;
    auto whole = [&](const void *base, int64_t ld2) { return n + 4 <= N && (((uintptr_t)base + (uintptr_t)((m * ld2 + n) * eb)) % (4 * eb)) == 0; };
    auto put = [&](void *base, int64_t ld2, const float (&v)[4]) {
        if (whole(base, ld2)) store_typed<4>(base, m * ld2 + n, e.type, v);
        else
            for (int j = 0; j < 4 && n + j < N; ++j) { const float o[1] = {v[j]}; store_typed<1>(base, m * ld2 + n + j, e.type, o); }
    };
    if (e.z) put(e.z, e.ldz, z);
    activate(z, e.act);
    if (e.residual) {
        float r[4] = {0, 0, 0, 0};
        if (whole(e.residual, e.ldr)) load_typed<4>(r, e.residual, m * e.ldr + n, e.type);
        else
            for (int j = 0; j < 4 && n + j < N; ++j) { float o[1]; load_typed<1>(o, e.residual, m * e.ldr + n + j, e.type); r[j] = o[0]; }
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] += r[j];
    }
    put(e.y, e.ldy, z);
}

// Rows of any start and distance to rows that start on 16 bytes: 16 bytes per thread.
template <typename T>
__global__ void __launch_bounds__(256) pack_kernel(const T *__restrict__ src, int64_t ld, int64_t rows, int64_t len, T *__restrict__ dst, int64_t ldDst)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t perRow = ldDst / V, total = rows * perRow;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / perRow, c = (i - r * perRow) * V;
        Pack<T, V> v;
#pragma unroll
        for (int j = 0; j < V; ++j) v.v[j] = c + j < len ? src[r * ld + c + j] : T(0);
        *reinterpret_cast<Pack<T, V> *>(dst + r * ldDst + c) = v;
    }
}

// The waits of the product and of the norm's ring for copies that nobody makes: either one has to run out for every thread, and the one
// behind it at once; all of it in the status word, or that it went otherwise.
__global__ void __launch_bounds__(64) operator_wait_selftest_kernel(int32_t *status)
{
    __shared__ Shared sh;
    __shared__ RingShared ring;
    if (threadIdx.x == 0) {
        for (int k = 0; k < 2; ++k) {
            mbar_init(&sh.full[k], 1);
            mbar_init(&ring.bar[0][k], 1);
        }
        sh.abort = 0;
        ring.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const bool came = warp_wait_for(&sh.full[0], 0, &sh, 1u << 5) || ring_wait(&ring.bar[0][0], 0, &ring, 1u << 12);
    const bool then = warp_wait_for(&sh.full[1], 0, &sh) || ring_wait(&ring.bar[0][1], 0, &ring);
    const bool wrong = __syncthreads_or(came || then);
    if (threadIdx.x == 0) atomicOr(status, wrong || !sh.abort || !ring.abort ? kDevBadState : kDevTimeout);
}

// ---- host side ----

struct Plan {
    bool pair;
    int tn, splits, slabsPerSplit;
    int64_t slabs, tilesM, tilesN, rowsPart, ldPart;     // rowsPart: whole pieces of 32 rows, which are stored whole
    bool packA, packB;
    int64_t ldA, ldB;
    size_t partAt, aAt, bAt, bytes;
};

bool mappable(const Operand &o, int64_t eb) { return ((uintptr_t)o.p) % 16 == 0 && o.ld * eb % 16 == 0 && o.ld * eb < (1LL << 40); }

// Which tile, and into how many pieces the k axis is cut: the least of an estimate in cycles.  A slab costs an SM its share of the
// tensor pipe (128 x 256 x 128 bytes: 512 cycles) or what its operands take from L2 (some 56 bytes a cycle), a tile its epilogue behind the
// last slab; pieces cost the join's launch and their way through L2.
Plan make_plan(const rcd_ctx *ctx, const Product &p, bool packA, bool packB)
{
    Plan best{};
    const int64_t eb = elem_bytes(p.type);
    best.packA = packA;
    best.packB = packB;
    const int64_t slabElems = kSlab / eb;
    const int64_t slabs = (p.K + slabElems - 1) / slabElems;
    double least = 1e300;
    for (int pair = 0; pair < 2; ++pair)
        for (int tn = 64; tn <= 256; tn += 64) {
            if (pair && p.b.across && tn % 128 != 0) continue;         // (boxes of 64 columns per CTA)
            if (pair && ctx->smCount < 2) continue;
            const int64_t tilesM = (p.M + (pair ? 256 : 128) - 1) / (pair ? 256 : 128), tilesN = (p.N + tn - 1) / tn;
            const int64_t slots = pair ? ctx->smCount / 2 : ctx->smCount, tiles = tilesM * tilesN;
            if (tiles > 0x3fffffffLL) continue;
            const double slab = std::max(512.0 * tn / 256.0, (pair ? 128.0 + tn / 2 : 128.0 + tn) * kSlab / 56.0) + 10.0;
            for (int splits = 1; splits <= 64; ++splits) {
                if (splits > 1 && (tiles * splits > 2 * slots || splits > slabs)) break;
                const int64_t per = (slabs + splits - 1) / splits;
                if (splits > 1 && (splits - 1) * per >= slabs) continue;     // (an empty piece)
                const int64_t waves = (tiles * splits + slots - 1) / slots;
                double t = (double)waves * (double)per * slab + 2500.0 + 9.0 * tn;
                if (splits > 1) t += 6000.0 + (double)p.M * (double)p.N * 8.0 * splits / 5000.0;
                if (t < least) {
                    least = t;
                    best.pair = pair != 0;
                    best.tn = tn;
                    best.splits = splits;
                    best.slabsPerSplit = (int)per;
                    best.slabs = slabs;
                    best.tilesM = tilesM;
                    best.tilesN = tilesN;
                }
            }
        }
    size_t at = 0;
    best.ldPart = (p.N + 31) / 32 * 32;
    best.rowsPart = (p.M + 31) / 32 * 32;
    if (best.splits > 1) at += align_up((size_t)(best.splits * best.rowsPart * best.ldPart) * 4);
    auto pack = [&](const Operand &o, int64_t mn, bool wanted, int64_t *ld, size_t *where) {
        const int64_t rows = o.across ? p.K : mn, len = o.across ? mn : p.K, v = 16 / eb;
        *ld = wanted ? (len + v - 1) / v * v : o.ld;
        *where = at;
        if (wanted) at += align_up((size_t)(rows * *ld * eb));
    };
    pack(p.a, p.M, best.packA, &best.ldA, &best.aAt);
    pack(p.b, p.N, best.packB, &best.ldB, &best.bAt);
    best.bytes = at;
    return best;
}

// A call asks three times (workspace twice, launch), a program the same sizes over and over: the last eight answers are kept, by
// sizes, types and orders alone.
struct PlanCache {
    struct Entry { int64_t M, N, K, ldA, ldB; int how; Plan plan; } of[8];
    unsigned next;
};
const Plan &plan_product(rcd_ctx *ctx, const Product &p)
{
    static_assert(sizeof(PlanCache) <= sizeof(ctx->productPlans) && std::is_trivially_copyable<PlanCache>::value, "the context has room for it");
    PlanCache &c = *reinterpret_cast<PlanCache *>(ctx->productPlans);      // (zeros at first: how 0 is nobody's)
    const int64_t eb = elem_bytes(p.type);
    const bool packA = !mappable(p.a, eb), packB = !mappable(p.b, eb);
    const int how = 1 | (int)p.type << 1 | (int)p.a.across << 3 | (int)p.b.across << 4 | (int)packA << 5 | (int)packB << 6;
    for (const PlanCache::Entry &e : c.of)
        if (e.how == how && e.M == p.M && e.N == p.N && e.K == p.K && e.ldA == p.a.ld && e.ldB == p.b.ld) return e.plan;
    PlanCache::Entry &e = c.of[c.next++ % 8];
    e = {p.M, p.N, p.K, p.a.ld, p.b.ld, how, make_plan(ctx, p, packA, packB)};
    return e.plan;
}

rcd_status encode(rcd_ctx *ctx, CUtensorMap *map, CUtensorMapDataType type, const void *p, int64_t inner, int64_t outer, int64_t ldBytes, int boxInner, int boxOuter)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(ctx, RCD_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    const cuuint64_t strides[1] = {(cuuint64_t)ldBytes};
    const cuuint32_t box[2] = {(cuuint32_t)boxInner, (cuuint32_t)boxOuter};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult cr = fn(map, type, 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (cr != CUDA_SUCCESS) return fail(ctx, RCD_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)cr);
    return RCD_OK;
}
CUtensorMapDataType map_type(rcd_elem t)
{
    return t == RCD_ELEM_I8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : t == RCD_ELEM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
           : t == RCD_ELEM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
}

template <typename Kernel>
rcd_status run_product(rcd_ctx *ctx, Kernel *kernel, int bit, int grid, size_t smem, const CUtensorMap (&maps)[5], const TcParams &q, cudaStream_t st)
{
    if (!(ctx->productReady >> bit & 1)) {              // (shared memory beyond 48 KB is asked for once per context and kernel)
        RCD_CUDA(ctx, allow_shared(kernel, kMostShared));
        ctx->productReady |= 1u << bit;
    }
    kernel<<<grid, kThreads, smem, st>>>(maps[0], maps[1], maps[2], maps[3], maps[4], q);
    ctx->kernelLaunches++;
    ctx->tcLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

}  // namespace

rcd_status launch_operator_wait_selftest(rcd_ctx *ctx, int32_t *status, cudaStream_t st)
{
    operator_wait_selftest_kernel<<<1, 64, 0, st>>>(status);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

size_t product_workspace(rcd_ctx *ctx, const Product &p) { return few_rows(p) ? 0 : plan_product(ctx, p).bytes; }

rcd_status launch_product(rcd_ctx *ctx, const Product &p, void *workspace, cudaStream_t st)
{
    if (few_rows(p)) return launch_few_rows(ctx, p, st);
    const Plan plan = plan_product(ctx, p);
    unsigned char *ws = (unsigned char *)workspace;
    const int64_t eb = elem_bytes(p.type);
    const bool i8 = p.type == RCD_ELEM_I8;
    auto operand = [&](const Operand &o, int64_t mn, bool pack, int64_t ld, size_t at, int boxRows, CUtensorMap *map) {
        const int64_t rows = o.across ? p.K : mn, len = o.across ? mn : p.K;
        const void *from = o.p;
        if (pack) {
            const unsigned grid = (unsigned)std::min<int64_t>((rows * (ld * eb / 16) + 255) / 256, (int64_t)ctx->smCount * 16);
            if (i8) pack_kernel<int8_t><<<grid, 256, 0, st>>>((const int8_t *)o.p, o.ld, rows, len, (int8_t *)(ws + at), ld);
            else pack_kernel<uint16_t><<<grid, 256, 0, st>>>((const uint16_t *)o.p, o.ld, rows, len, (uint16_t *)(ws + at), ld);
            ctx->kernelLaunches++;
            RCD_CUDA(ctx, cudaGetLastError());
            from = ws + at;
        }
        return encode(ctx, map, map_type(p.type), from, len, rows, ld * eb, o.across ? 64 : (int)(kSlab / eb), o.across ? kSlabRows16 : boxRows);
    };
    CUtensorMap maps[5] = {};
    RCD_TRY(operand(p.a, p.M, plan.packA, plan.ldA, plan.aAt, kRows, &maps[0]));
    RCD_TRY(operand(p.b, p.N, plan.packB, plan.ldB, plan.bAt, plan.pair ? plan.tn / 2 : plan.tn, &maps[1]));

    TcParams q{};
    q.M = (int32_t)p.M; q.N = (int32_t)p.N;
    q.tilesN = (int32_t)plan.tilesN;
    q.tiles = (int32_t)(plan.tilesM * plan.tilesN);
    q.units = q.tiles * plan.splits;
    q.slabs = (int32_t)plan.slabs;
    q.slabsPerSplit = plan.slabsPerSplit;
    q.tn = plan.tn;
    const int chunk = p.out.type == RCD_ELEM_F32 ? kChunkSlabs : kChunkSlabs16;
    const bool chunks = !i8 && plan.slabsPerSplit > (p.out.type == RCD_ELEM_F32 ? chunk : 2 * chunk);
    q.chunk = chunks ? chunk : q.slabs;
    q.stageBytes = kABytes + (plan.pair ? plan.tn / 2 : plan.tn) * kSlab;
    q.stages = std::min(kMostStages, (kMostShared - kFixedShared) / q.stageBytes);
    q.idesc = (i8 ? (2u << 4) | (1u << 7) | (1u << 10)                                     // S8 x S8 -> S32
                  : (1u << 4) | (p.type == RCD_ELEM_BF16 ? (1u << 7) | (1u << 10) : 0u)) | // BF16 x BF16 or F16 x F16 -> F32
              (p.a.across ? 1u << 15 : 0u) | (p.b.across ? 1u << 16 : 0u) | ((uint32_t)(plan.tn >> 3) << 17) | ((uint32_t)((plan.pair ? 256 : 128) >> 4) << 24);
    q.e = p.out;
    q.raw = plan.splits > 1;
    if (q.raw) {
        q.e = Epilogue{};
        q.e.type = RCD_ELEM_F32;
        q.e.y = ws + plan.partAt;
        q.e.ldy = plan.ldPart;
        q.rowsPart = (int32_t)plan.rowsPart;
    }
    q.status = ctx->statusOwn + kOperatorStatus;
    const int64_t yb = elem_bytes(q.e.type);
    auto output = [&](const void *base, int64_t ld, int64_t rows, bool *use, CUtensorMap *map) {
        *use = base && rows_aligned(base, ld, yb, 16) && ld * yb < (1LL << 40);
        return *use ? encode(ctx, map, map_type(q.e.type), base, q.raw ? plan.ldPart : p.N, rows, ld * yb, (int)(128 / yb), 32) : RCD_OK;
    };
    RCD_TRY(output(q.e.y, q.e.ldy, q.raw ? plan.splits * plan.rowsPart : p.M, &q.tmaY, &maps[2]));
    RCD_TRY(output(q.e.z, q.e.ldz, p.M, &q.tmaZ, &maps[3]));
    RCD_TRY(output(q.e.residual, q.e.ldr, p.M, &q.tmaR, &maps[4]));
    q.edgeByHand = !q.raw && p.N * yb % 16 != 0;           // (a piece of the k axis has rows of whole 128 bytes)
    const size_t smem = (size_t)q.stages * q.stageBytes + kFixedShared;
    const int slots = plan.pair ? ctx->smCount / 2 : ctx->smCount;
    const int grid = std::min(slots, q.units) * (plan.pair ? 2 : 1);
    const int order = i8 ? 0 : !p.a.across && !p.b.across ? 1 : !p.a.across ? 2 : 3;
    if (p.a.across && !p.b.across) return fail(ctx, RCD_ERR_INTERNAL, "no product takes these orders");
    auto run = [&](auto *single, auto *pair, int bit) { return plan.pair ? run_product(ctx, pair, bit, grid, smem, maps, q, st) : run_product(ctx, single, bit + 1, grid, smem, maps, q, st); };
    const int wide = !chunks ? 0 : q.e.type == RCD_ELEM_F32 ? 32 : 64;
    auto run_order = [&](auto acrossA, auto acrossB, int bit) {
        constexpr bool kA = decltype(acrossA)::value, kB = decltype(acrossB)::value;
        return wide == 0    ? run(product_kernel<false, kA, kB>, product_pair_kernel<false, kA, kB>, bit)
               : wide == 32 ? run(product_kernel<false, kA, kB, 32>, product_pair_kernel<false, kA, kB, 32>, bit + 2)
                            : run(product_kernel<false, kA, kB, 64>, product_pair_kernel<false, kA, kB, 64>, bit + 4);
    };
    const std::false_type along;
    const std::true_type across;
    const rcd_status rs = order == 0   ? run(product_kernel<true, false, false>, product_pair_kernel<true, false, false>, 0)
                          : order == 1 ? run_order(along, along, 2)
                          : order == 2 ? run_order(along, across, 8)
                                       : run_order(across, across, 14);
    if (rs != RCD_OK || !q.raw) return rs;
    const int64_t threads = p.M * ((p.N + 3) / 4);
    if (i8) join_kernel<true><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(ws + plan.partAt, plan.splits, (int32_t)p.M, plan.rowsPart, (int32_t)p.N, plan.ldPart, p.out);
    else join_kernel<false><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(ws + plan.partAt, plan.splits, (int32_t)p.M, plan.rowsPart, (int32_t)p.N, plan.ldPart, p.out);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

}  // namespace rcd

// The product on the tensor cores that rcd_linear, the loss of a head and the orthogonalised update share:  C = A B^T, finished in one of several
// forms (see Form).
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
// Warp roles: 0 = TMA producer, 1 = TMEM allocation + MMA issue, 4..11 = epilogue, two per quarter of the TMEM lanes.
// Every wait is bounded, as in the similarity kernel: on expiry the CTA records kDevTimeout and leaves.
#pragma once

#include "rcd_act.cuh"
#include "rcd_linear.h"
#include "rcd_tc.cuh"
#include "rcd_walk.h"

namespace rcd {

constexpr int kRows = kOperandRows, kSlab = kOperandSlab, kMostStages = kOperandStages, kMostShared = kBlockShared;
constexpr int kSlabRows16 = 64;                         // k elements of 16 bits per slab
constexpr int kBox = 64 * kSlab;                        // 8 KB: 64 k rows of 64 elements
constexpr int kEpiWarps = 8;
// The tensor cores cut an fp32 sum off where they cannot hold it, towards zero: products of fp16 and of one sign lose 6.5e-9 of the result
// each, 3.2e-4 over 50 000 (two thirds of the type's half step).  So sums are taken in chunks that are added up outside with rounding.
// fp32 outputs: 512 k (2.4e-6 within a chunk, bf16 2.3e-7, and half a unit of fp32 at most for each of them).  16-bit outputs: 2048 k (1.3e-5)
// where a piece has more than 4096, up to which the loss is a twentieth of fp16's half step.  (Gradients of 2048 x 2048 weights over 600 000
// rows: 3.56 ms in chunks, 3.45 in one sum.)
// Logits whose gradients are summed over the rows in fp32 (a head's dbias, where p and the labels nearly cancel, and what all rows' z have lost adds up): 128 k, which from some 1000
// classes on is as exact as fp32 products.  Of 5000 x 2048 over 1000 classes dbias is 1.5e-5 off in one sum, 3.3e-6 in chunks of 512, 1.6e-6 of 256, 7.8e-7 of 128, 4.3e-7 of 64 (fp32
// products 8.4e-7); the call takes 89, 98, 102, 106 and 119 us.  What is left comes from the chunks: with exp to the last bit it is the same.  The loss adds up 512 k; its lse is 2e-6 low,
// and dbias from it 2.7e-6 off the loss's own gradient.  (With chunks of 128 in the loss, too, 2e-7; but 5000 x 2048 over 1000 classes would take 40 us for 30 there, and 8192 x 4096 over
// 32 768 2.15 ms for 1.46.)  Fewer classes have larger p, which lose more: 20 000 x 2048 over ten in chunks of 128 4.5e-6 off, and 1.5e-5 with the loss's lse.  Where one tile has them
// all (kOneTile) the logits are the loss's, in chunks of 512, and p is brought to a sum of one: 5.2e-7 and 5.4e-7 (111 us for 117).
constexpr int kChunkSlabs = 8, kChunkSlabs16 = 32, kChunkSlabsSums = 2;
constexpr int kFirstEpiWarp = 4;                        // (a warpgroup for the two that issue: registers are handed over by warpgroups)
constexpr int kThreads = 32 * (kFirstEpiWarp + kEpiWarps);
// Registers per thread at launch (65536 over 12 warps in whole eights), and how the warpgroups split them: 128 x 40 + 256 x 232 = 384 x 168.  (With 168 for all, sums of
// chunks leave the registers at their ends: gradients of 5000 x 2048 over 1000 classes 100 us for 98, of 8192 x 4096 over 8192 with dbias 1257 for 1232.)
constexpr int kLaunchRegs = 168, kIssueRegs = 40, kEpiRegs = 232;
static_assert(128 * kIssueRegs + 32 * kEpiWarps * kEpiRegs <= kThreads * kLaunchRegs, "what one warpgroup gets the other has to have given");
constexpr int kPiece = 32 * 128;                        // an epilogue warp's piece of the output: 32 rows of 128 bytes
constexpr int kColumnBytes = kEpiWarps * 2 * 128 * 4;   // a warp's 128 columns of a tile: biases and scales
constexpr uint32_t kWaitTurns = 1u << 16;               // of at most 20 us: a second or so

struct __align__(8) ProductShared {
    uint64_t full[kMostStages], empty[kMostStages];     // full: CTA 0's of a pair
    uint64_t accFull[2], accEmpty[2];                   // accEmpty: CTA 0's of a pair
    uint64_t residual[kEpiWarps][2];
    uint64_t handed[4][2];                              // kLoss: the quarter's second warp has left its half of a tile, two tiles in turn; kOneTile: both have
    uint32_t tmemBase;
    int32_t abort;
};
constexpr int kFixedShared = (int)sizeof(ProductShared);
constexpr int kJoinStaging = 2 * 4 * 3 * 32 * 4;        // kLoss: what the second warp of a quarter hands to the first, two tiles in turn

struct TcParams {
    int32_t M, N, units, slabs, slabsPerSplit, chunk, tn, stages, stageBytes, stagingBytes, columnBytes, places, aRows, rowsPart;
    uint32_t idesc;
    Walk walk;
    int32_t aStep, bStep, yStep, rStep;                        // rows from one matrix of a batch to the next (rows of k, where an operand is across)
    Epilogue e;
    Head head;
    Scaling s;
    bool raw;                                           // accumulators as they are, into e.y: [split][rowsPart][ldy]
    bool tmaY, tmaZ, tmaR, edgeByHand;                  // edgeByHand: a piece that holds the rows' ends, since TMA stores 16 bytes at a time
    int32_t *status;
};

// (Suspended by the hardware up to 20 us at a time: polls with pauses cost the ring half a slab's time at every turn.)
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, ProductShared *sh, uint32_t turns = kWaitTurns)
{
    for (uint32_t turn = 0; turn < turns; ++turn) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
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
__device__ __forceinline__ bool warp_wait_for(uint64_t *bar, uint32_t parity, ProductShared *sh, uint32_t turns = kWaitTurns)
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

__device__ __forceinline__ void copy_float(float *to, const float *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(smem_addr(to)), "l"(from) : "memory");
}

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
    if constexpr (!kLoad && sizeof(T) == 2) {
        // A whole piece: two elements in a store wherever a row starts, eight rows at a time and no lane by itself.  (5003 x 64 x 1001: element by element 33 us.)
        if (rows == 32 && cols >= kCols) {
            const uint32_t *const words = reinterpret_cast<const uint32_t *>(piece);
            for (int r0 = 0; r0 < 32; r0 += 8, at += 8 * ld) {
                uint32_t w[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) w[r] = words[(piece_at(r0 + r, lane >> 2) >> 2) + (lane & 3)];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    T *const row = at + r * ld;
                    const uint32_t next = __shfl_down_sync(0xffffffffu, w[r], 1);
                    if ((uintptr_t)row & 2) {
                        // elements 1 and 2, 3 and 4, ...; the first and the last by themselves
                        if (lane < 31) *reinterpret_cast<uint32_t *>(row + 2 * lane + 1) = __byte_perm(w[r], next, 0x5432);
                        if (lane == 0 || lane == 31) row[lane ? kCols - 1 : 0] = (T)(lane ? w[r] >> 16 : w[r]);
                    } else {
                        *reinterpret_cast<uint32_t *>(row + 2 * lane) = w[r];
                    }
                }
            }
            return;
        }
    }
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
// v += factor * row (factor 1: the sum itself, rounded once)
__device__ __forceinline__ void add_row(const unsigned char *piece, int row, int chunk, float (&v)[32], rcd_elem type, float factor)
{
    if (type == RCD_ELEM_F32) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float4 x = *reinterpret_cast<const float4 *>(piece + piece_at(row, c));
            v[4 * c] = fmaf(factor, x.x, v[4 * c]);
            v[4 * c + 1] = fmaf(factor, x.y, v[4 * c + 1]);
            v[4 * c + 2] = fmaf(factor, x.z, v[4 * c + 2]);
            v[4 * c + 3] = fmaf(factor, x.w, v[4 * c + 3]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint4 x = *reinterpret_cast<const uint4 *>(piece + piece_at(row, chunk + c));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2(w[i], type);
                v[8 * c + 2 * i] = fmaf(factor, f.x, v[8 * c + 2 * i]);
                v[8 * c + 2 * i + 1] = fmaf(factor, f.y, v[8 * c + 2 * i + 1]);
            }
        }
    }
}
// The log of a sum of exponentials in pieces: a finite reference `top` and the sum of exp(z - top).  Values of -infinity add nothing and NaN
// stays; +infinity leaves the largest finite number as the reference and an infinite sum.
struct SumOfExp { float top, sum; };
constexpr float kLargest = 3.402823466e38f;
__device__ __forceinline__ SumOfExp no_terms() { return {-kLargest, 0.0f}; }
__device__ __forceinline__ void add_terms(SumOfExp &s, const float (&z)[32])
{
    float m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = fmaxf(fmaxf(z[j], z[j + 8]), fmaxf(z[j + 16], z[j + 24]));
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = fmaxf(m[j], m[j + 4]);
    const float top = fminf(fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), s.top), kLargest);
    // (the difference first: digits of z that exp(z - top) depends on are still there at large z)
    const Two less = two(-top, -top), log2e = two(kLog2e, kLog2e);
    Two sum[4];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float2 a = parts(mul2(add2(two(z[2 * j], z[2 * j + 1]), less), log2e));
        const Two e = two(exp2_fast(a.x), exp2_fast(a.y));
        sum[j & 3] = j < 4 ? e : add2(sum[j & 3], e);
    }
    const float2 both = parts(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
    s.sum = fmaf(s.sum, exp2_fast((s.top - top) * kLog2e), both.x + both.y);
    s.top = top;
}
__device__ __forceinline__ void join_terms(SumOfExp &s, const SumOfExp &o)
{
    const float top = fmaxf(s.top, o.top);
    s.sum = s.sum * exp2_fast((s.top - top) * kLog2e) + o.sum * exp2_fast((o.top - top) * kLog2e);
    s.top = top;
}

// A row's loss from its sum and its label's logit.
__device__ __forceinline__ void finish_loss(const SumOfExp &s, int32_t label, int32_t classes, float picked, float *loss, float *lse, int32_t *status)
{
    const float all = s.top + logf(s.sum);
    if (lse) *lse = all;
    const bool beyond = label >= classes;
    if (beyond) atomicOr(status, kDevBadLabel);
    *loss = beyond ? NAN : label < 0 ? 0.0f : all - picked;
}

// Sums of 32 columns over the warp's 32 rows, a lane's row in v: lane j ends with column j's, added up in the rows' order by fours.  Through 4 KB of
// shared memory, a word of row r and column c at 32 r + (c ^ r): lanes meet no other's bank on either way.
__device__ __forceinline__ float column_sum(const float (&v)[32], float *place)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 32; ++j) place[32 * lane + (j ^ lane)] = v[j];
    __syncwarp();
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 32; ++r) sum[r & 3] += place[32 * r + (lane ^ r)];
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// kChunks: 0, or the columns of a piece of the output, whose sums are taken in chunks.
template <Form kForm, bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks, bool kPair>
__device__ __forceinline__ void product_body(const CUtensorMap &mapA, const CUtensorMap &mapB, const CUtensorMap &mapY, const CUtensorMap &mapZ, const CUtensorMap &mapR, const TcParams &p)
{
    constexpr bool kIsScaled = kForm == kScaled || kForm == kScaledLow, kIsGrads = kForm == kLogitGrads || kForm == kOneTile;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char *const tiles = smem;
    unsigned char *const staging = smem + (size_t)p.stages * p.stageBytes;
    float *const columns = reinterpret_cast<float *>(staging + p.stagingBytes);
    ProductShared &sh = *reinterpret_cast<ProductShared *>(staging + p.stagingBytes + p.columnBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kPair ? (int)(blockIdx.x & 1) : 0;
    const int first = kPair ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, step = kPair ? (int)(gridDim.x >> 1) : (int)gridDim.x;

    if (warp == 2 && elect_one()) {
        for (const CUtensorMap *map : {&mapA, &mapB, &mapY, &mapR}) asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMostStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&sh.accFull[b], 1); mbar_init(&sh.accEmpty[b], (kPair ? 2 : 1) * kEpiWarps); }
        for (int w = 0; w < kEpiWarps; ++w) { mbar_init(&sh.residual[w][0], 1); mbar_init(&sh.residual[w][1], 1); }
        for (int w = 0; w < 4; ++w) { mbar_init(&sh.handed[w][0], kForm == kOneTile ? 2 : 1); mbar_init(&sh.handed[w][1], kForm == kOneTile ? 2 : 1); }
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
    after_the_one_before();
    const uint32_t tmemBase = sh.tmemBase;
    const int rowsPerTile = kPair ? 2 * kRows : kRows;
    const int nMine = kPair ? p.tn / 2 : p.tn;           // B's rows that this CTA brings in

    if (warp < kFirstEpiWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kIssueRegs));
    if (warp == 0) {
        // ---------------- TMA producer ----------------
        // (The whole warp goes through the loop, one lane issues: addresses stay in uniform registers, which is where these instructions
        // want them.  With the loop inside one lane's branch a slab took the issuer 600 cycles whatever its size.)
        const bool leader = elect_one();
        int s = 0;
        uint32_t phase = 1;
        bool ok = true;
        const int slabElems = kInt8 ? kSlab : kSlab / 2;
        const uint32_t bytes = (uint32_t)(kPair ? 2 : 1) * (uint32_t)((p.aRows + nMine) * kSlab);
        for (int u = first; u < p.units && ok; u += step) {
            const Unit t = unit_of(p.walk, u);
            const int m0 = t.m * rowsPerTile + rank * kRows, n0 = t.n * p.tn + rank * nMine;
            const int aRow = kIsScaled ? t.batch * p.aStep : 0, bRow = kIsScaled ? t.batch * p.bStep : 0;
            const int end = min(p.slabs, (t.split + 1) * p.slabsPerSplit);
            for (int kb = t.split * p.slabsPerSplit; kb < end; ++kb) {
                if (!warp_wait_for(&sh.empty[s], phase, &sh)) { ok = false; break; }
                unsigned char *a = tiles + s * p.stageBytes, *b = a + p.aRows * kSlab;
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
                        for (int j = 0; j < kRows / 64; ++j) load(a + j * kBox, &mapA, m0 + 64 * j, aRow + kb * kSlabRows16);
                    } else {
                        load(a, &mapA, kb * slabElems, aRow + m0);
                    }
                    if constexpr (kAcrossB) {
                        for (int j = 0; j < nMine / 64; ++j) load(b + j * kBox, &mapB, n0 + 64 * j, bRow + kb * kSlabRows16);
                    } else {
                        load(b, &mapB, kb * slabElems, bRow + n0);
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
                const Unit t = unit_of(p.walk, u);
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
                        const uint32_t aAddr = tile0 + (uint32_t)(s * p.stageBytes), bAddr = aAddr + (uint32_t)(p.aRows * kSlab);
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
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kEpiRegs));
        // ---------------- epilogue: this CTA's 128 rows ----------------
        const int q = warp & 3, ew = warp - kFirstEpiWarp, half = ew >> 2;       // TMEM lanes 32 q ..; pieces half, half + 2, ...
        unsigned char *const mine = staging + ew * p.places * kPiece;
        float *const biases = columns + ew * 256, *const scales = biases + 128;
        const Epilogue &e = p.e;
        const int wide = kChunks ? kChunks : e.type == RCD_ELEM_F32 ? 32 : 64;        // columns of a piece
        const int pieces = p.tn / wide;
        // a piece's coordinates; false where nothing of it lies inside the output
        struct Piece { int row, col, base, from; };        // base, from: rows of the output and of the residual before this matrix
        auto piece_of = [&](const Unit &t, int k, Piece *o) {
            o->row = t.m * rowsPerTile + rank * kRows + q * 32;
            o->col = t.n * p.tn + k * wide;
            o->base = kIsScaled ? t.batch * p.yStep : 0;
            o->from = kIsScaled ? t.batch * p.rStep : 0;
            return o->row < p.M && o->col < p.N;
        };
        // the residual of the next piece that has one, from piece k of t, which is unit u, on, is on its way into buffer `to`
        auto fetch = [&](Unit t, int u, int k, int to) {
            Piece o;
            while (true) {
                for (; k < pieces; k += 2)
                    if (piece_of(t, k, &o)) {
                        mbar_expect_tx(&sh.residual[ew][to], kPiece);
                        tma_load_2d(mine + to * kPiece, &mapR, o.col, o.from + o.row, &sh.residual[ew][to]);
                        return;
                    }
                if ((u += step) >= p.units) return;
                t = unit_of(p.walk, u);
                k = half;
            }
        };
        const bool mirrors = kIsScaled && p.walk.subM != 0;
        const bool sums = kIsGrads && p.head.sums != nullptr;
        const bool alternate = p.places == 2 && e.z == nullptr && !mirrors && !sums;      // two places in turn, or one for y and one for z, the transpose or sums; or only the one
        uint32_t nt = 0, turn = 0;
        [[maybe_unused]] uint32_t tile = 0;
        if (p.tmaR && lane == 0 && first < p.units) fetch(unit_of(p.walk, first), first, half, 0);
        bool ok = true;
        unsigned char *yPiece = mine;
        unsigned char *const zPiece = mine + kPiece;
        // a piece's place in shared memory is free, and the residual lies there
        auto begin_piece = [&](const Unit &t, int u, int k, const Piece &o) {
            yPiece = mine + (alternate ? (turn & 1) * kPiece : 0);
            // (what was stored from it has been read out of it; a residual that comes next needs the other place too)
            if (lane == 0) {
                if (alternate && !p.tmaR) bulk_wait_read<1>();
                else bulk_wait_read<0>();
            }
            __syncwarp();
            if (p.tmaR) {
                if (alternate && lane == 0) fetch(t, u, k + 2, (turn & 1) ^ 1);
                // (with z in the other buffer the residual is fetched when the last piece has left)
                return warp_wait_for(&sh.residual[ew][alternate ? turn & 1 : 0], alternate ? (turn >> 1) & 1 : turn & 1, &sh);
            }
            if (e.residual) {
                const int64_t at = ((int64_t)o.from + o.row) * e.ldr + o.col;
                if (e.type == RCD_ELEM_F32) move_piece<true>(yPiece, (float *)e.residual + at, e.ldr, p.M - o.row, p.N - o.col);
                else move_piece<true>(yPiece, (uint16_t *)e.residual + at, e.ldr, p.M - o.row, p.N - o.col);
                __syncwarp();
            }
            return true;
        };
        // The biases and scales of the warp's columns of a tile (up to four times 32), on their way into shared memory while the tile is computed.
        const bool anyColumns = !p.raw && (e.bias || (kInt8 && e.ws));
        auto ask_columns = [&](const Unit &t) {
            if (!anyColumns) return;
            __syncwarp();                                              // (all have read the last tile's)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int col = t.n * p.tn + (wide == 64 ? (half + 2 * (c >> 1)) * 64 + (c & 1) * 32 : (half + 2 * c) * 32) + lane;
                if (col < p.N) {
                    if (e.bias) copy_float(biases + c * 32 + lane, e.bias + col);
                    if (kInt8 && e.ws) copy_float(scales + c * 32 + lane, e.ws + col);
                }
            }
        };
        auto have_columns = [&] {
            if (!anyColumns) return;
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
        };
        // What the lane's row brings along: asked for when the tile before is about to be finished, worked out when its own comes.
        struct Asked { int label; float sx, lse, dloss, dlse; };
        auto ask_row = [&](const Unit &t) {
            Asked r{-1, 1.0f, 0.0f, 0.0f, 0.0f};
            const int row = t.m * rowsPerTile + rank * kRows + q * 32 + lane;
            if (row < p.M) {
                if constexpr (kInt8) {
                    if (e.xs) r.sx = e.xs[row];
                }
                if constexpr (kForm == kLoss || kIsGrads) r.label = p.head.labels[row];
                if constexpr (kIsGrads) {
                    r.lse = p.head.lse[row];
                    r.dloss = p.head.dloss ? p.head.dloss[row] : 1.0f;
                    if (p.head.dlse) r.dlse = p.head.dlse[row];
                }
            }
            return r;
        };
        struct Row {
            float sx;                                                  // int8: its scale
            int label;                                                 // its class's column in this output
            float lse, weight, atLabel;                                // kLogitGrads: dz = weight * p, less atLabel in the label's column
            float alpha, beta;                                         // kScaled
            bool mirror;
        };
        [[maybe_unused]] const float up = kIsGrads && p.head.up ? *p.head.up : 1.0f;
        auto row_of = [&](const Unit &t, const Asked &asked) {
            Row r{};
            r.sx = asked.sx;
            if constexpr (kForm == kLoss || kIsGrads) {
                const bool valid = asked.label >= 0 && asked.label < p.head.classes;
                r.label = valid ? asked.label - p.head.firstClass : -1;          // (another piece's: outside 0..N-1)
                if constexpr (kIsGrads) {
                    if (asked.label >= p.head.classes && t.n == 0) atomicOr(p.status, kDevBadLabel);
                    const float g = valid ? asked.dloss : 0.0f;
                    r.lse = asked.lse == -INFINITY ? INFINITY : asked.lse;         // (a row without a class that is open: p is 0)
                    r.weight = (g + asked.dlse) * up;
                    r.atLabel = g * up;
                }
            }
            if constexpr (kIsScaled) {
                const Scaling &sc = p.s;
                const float f = sc.factor ? sc.factor[t.batch] : 1.0f;
                auto power = [&](int n) { return n == 0 ? 1.0f : n == 1 ? f : f * f; };
                r.alpha = sc.alpha * power(sc.alphaPower);
                r.beta = sc.beta * power(sc.betaPower);
                r.mirror = t.mirror;
            }
            return r;
        };
        // kLogitGrads: the logits of 32 columns to exp(z - lse)
        [[maybe_unused]] auto exponentials = [&](float (&z)[32], float lse, int c) {
            if (e.bias) {
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 b = reinterpret_cast<const float4 *>(biases + c * 32)[j / 4];
                    z[j] += b.x; z[j + 1] += b.y; z[j + 2] += b.z; z[j + 3] += b.w;
                }
            }
            const Two less = two(-lse, -lse), log2e = two(kLog2e, kLog2e);
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                const float2 a = parts(mul2(add2(two(z[j], z[j + 1]), less), log2e));
                z[j] = exp2_fast(a.x);
                z[j + 1] = exp2_fast(a.y);
            }
        };
        // 32 columns of the lane's row, from column h of the piece on, the warp's c-th
        auto finish = [&](float (&z)[32], const Row &r, int h, int c, const Piece &o) {
            if (p.raw) {
                // (as they are)
            } else if constexpr (kIsScaled) {
#pragma unroll
                for (int j = 0; j < 32; ++j) z[j] *= r.alpha;
                if (e.residual) add_row(yPiece, lane, h / 8, z, p.s.residualType, r.beta);
                if (kForm == kScaledLow && o.row + lane < p.M) {       // (rows of whole 64s: straight from memory, in one product of an update)
                    const uint4 *const low = reinterpret_cast<const uint4 *>((const __half *)p.s.low + ((int64_t)o.from + o.row + lane) * e.ldr + o.col + h);
                    const float beta = r.beta * (1.0f / (1 << kLowUp));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint4 x = low[i];
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = unpack2(w[j], RCD_ELEM_F16);
                            z[8 * i + 2 * j] = fmaf(beta, f.x, z[8 * i + 2 * j]);
                            z[8 * i + 2 * j + 1] = fmaf(beta, f.y, z[8 * i + 2 * j + 1]);
                        }
                    }
                }
                if (r.mirror) {                                        // (rows of 64 bytes: a lane's row is a column there)
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const uint32_t two = pack2(z[j], z[j + 1], e.type);
                        *reinterpret_cast<uint16_t *>(zPiece + (h + j) * 64 + lane * 2) = (uint16_t)two;
                        *reinterpret_cast<uint16_t *>(zPiece + (h + j + 1) * 64 + lane * 2) = (uint16_t)(two >> 16);
                    }
                }
            } else if constexpr (kIsGrads) {
                exponentials(z, r.lse, c);
                const Two weight = two(r.weight, r.weight);
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    const float2 dz = parts(mul2(two(z[j], z[j + 1]), weight));
                    z[j] = dz.x;
                    z[j + 1] = dz.y;
                }
                const int at = r.label - (o.col + h);
                if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[j] -= at == j ? r.atLabel : 0.0f;
                }
                if (r.weight == 0.0f && r.atLabel == 0.0f) {           // (whatever p is: a row that is passed over may hold anything)
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[j] = 0.0f;
                }
            } else {
                if constexpr (kInt8) {
                    if (e.xs) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] *= r.sx;
                    }
                    if (e.ws) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 w = reinterpret_cast<const float4 *>(scales + c * 32)[j / 4];
                            z[j] *= w.x; z[j + 1] *= w.y; z[j + 2] *= w.z; z[j + 3] *= w.w;
                        }
                    }
                }
                if (e.bias) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 b = reinterpret_cast<const float4 *>(biases + c * 32)[j / 4];
                        z[j] += b.x; z[j + 1] += b.y; z[j + 2] += b.z; z[j + 3] += b.w;
                    }
                }
                if (e.z) put_row(zPiece, lane, h / 8, z, e.type);
                activate(z, e.act);
                if (e.residual) add_row(yPiece, lane, h / 8, z, e.type, 1.0f);
            }
            put_row(yPiece, lane, h / 8, z, e.type);
            if constexpr (kIsGrads) {
                if (p.head.sums) {
                    const float sum = column_sum(z, reinterpret_cast<float *>(zPiece)), down = 1.0f / up;           // (powers of two)
                    if (o.col + h + lane < p.N) p.head.sums[(int64_t)(o.row / 32) * p.N + o.col + h + lane] = sum * down;
                }
            }
        };
        auto end_piece = [&](const Unit &t, int u, int k, const Piece &o, int rowBase) {
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
            send(p.tmaY, &mapY, yPiece, e.y, e.ldy, rowBase + o.base);
            if (kIsScaled) {
                if (t.mirror && lane == 0) tma_store_2d(&mapZ, zPiece, o.row, o.base + o.col);
            } else if (e.z) {
                send(p.tmaZ, &mapZ, zPiece, e.z, e.ldz, 0);
            }
            if (lane == 0) bulk_commit();
            __syncwarp();
            if (p.tmaR && !alternate && lane == 0) {
                bulk_wait_read<0>();
                fetch(t, u, k + 2, 0);
            }
            ++turn;
        };
        // hands an accumulator back
        auto release = [&](uint32_t buf) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if constexpr (kPair) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(leader_addr(&sh.accEmpty[buf])) : "memory");
                else mbar_arrive(&sh.accEmpty[buf]);
            }
        };
        Unit next = first < p.units ? unit_of(p.walk, first) : Unit{};
        Asked askedNext = first < p.units ? ask_row(next) : Asked{};
        for (int u = first; u < p.units && ok; u += step) {
            const Unit t = next;
            const Asked asked = askedNext;
            if (u + step < p.units) next = unit_of(p.walk, u + step);
            const int rowBase = p.raw ? t.split * p.rowsPart : 0;
            const int row = t.m * rowsPerTile + rank * kRows + q * 32 + lane;
            const uint32_t lanes = (uint32_t)(q * 32) << 16;
            ask_columns(t);
            Row mineRow = row_of(t, asked);
            [[maybe_unused]] SumOfExp terms = no_terms();
            [[maybe_unused]] float picked = 0.0f;
            [[maybe_unused]] bool found = false;
            // kLoss: 32 columns join the row's sum, and its label's logit is noted
            [[maybe_unused]] auto take = [&](float (&z)[32], int c, const Piece &o) {
                if (e.bias) {
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 b = reinterpret_cast<const float4 *>(biases + c * 32)[j / 4];
                        z[j] += b.x; z[j + 1] += b.y; z[j + 2] += b.z; z[j + 3] += b.w;
                    }
                }
                if (o.col + 32 > p.N) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[j] = o.col + j < p.N ? z[j] : -INFINITY;
                }
                const int at = mineRow.label - o.col;
                if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) picked = at == j ? z[j] : picked;
                    found = found || (at >= 0 && at < 32);
                }
                add_terms(terms, z);
            };
            uint32_t buf = nt & 1;
            if constexpr (kChunks != 0) {
                // Sums of chunks (see kChunkSlabs) in a lane's 128 registers, four times 32 columns, while the next chunk is computed; what they come to goes back
                // into the last chunk's place and is finished from there as any accumulator.  (Finished from the registers, the code has four copies of what finishes 32 columns and
                // leaves the instruction cache, 2400 cycles for each; in a loop the sums leave the registers.)
                float sum[8][16];
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[i][j] = 0.0f;
                auto column = [&](int i) { return wide == 64 ? (half + 2 * (i >> 2)) * 64 + (i & 3) * 16 : (half + 2 * (i >> 1)) * 32 + (i & 1) * 16; };
                const int end = min(p.slabs, (t.split + 1) * p.slabsPerSplit);
#pragma unroll 1
                for (int begin = t.split * p.slabsPerSplit; begin < end; begin += p.chunk, ++nt) {
                    buf = nt & 1;
                    if (!warp_wait_for(&sh.accFull[buf], (nt >> 1) & 1, &sh)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // (columns behind the tile are loaded, too: nobody looks at them)
                        uint32_t v[16];
                        tmem_load_16cols(tmemBase + buf * 256 + lanes + (uint32_t)column(i), v);
                        tmem_load_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[i][j] += __uint_as_float(v[j]);
                    }
                    if (begin + p.chunk < end) release(buf);
                }
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < 8; ++i) tmem_store_16cols(tmemBase + buf * 256 + lanes + (uint32_t)column(i), sum[i]);
                tmem_store_wait();
            } else {
                if (!warp_wait_for(&sh.accFull[buf], (nt >> 1) & 1, &sh)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                ++nt;
            }
            have_columns();
            if (u + step < p.units) askedNext = ask_row(next);
            if constexpr (kForm == kOneTile) {
                // All classes are here, so p's sum is known: where it is one but for what the sums of other logits than lse's have lost, p is divided by it, and what is left in dbias is
                // what the classes have lost unlike one another.  Both warps of a quarter leave their half's sum and read the other's; the places are free again two tiles later,
                // since a warp is a tile ahead at most.
                float mass = 0.0f;
                for (int k = half; k < pieces; k += 2) {
                    Piece o;
                    if (!piece_of(t, k, &o)) continue;
                    for (int h = 0; h < wide; h += 32) {
                        uint32_t v[32];
                        tmem_load_32cols(tmemBase + buf * 256 + lanes + (uint32_t)(k * wide + h), v);
                        tmem_load_wait();
                        float z[32], some[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = __uint_as_float(v[j]);
                        exponentials(z, mineRow.lse, wide == 64 ? (k - half) + h / 32 : (k - half) / 2);
#pragma unroll
                        for (int j = 0; j < 32; ++j) some[j & 3] += o.col + h + j < p.N ? z[j] : 0.0f;
                        mass += (some[0] + some[1]) + (some[2] + some[3]);
                    }
                }
                const int at = 128 + (int)(tile & 1) * 32 + lane;      // (of the warp's columns, behind the biases)
                columns[ew * 256 + at] = mass;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.handed[q][tile & 1]);
                if (!warp_wait_for(&sh.handed[q][tile & 1], (tile >> 1) & 1, &sh)) { ok = false; break; }
                mass += columns[(ew ^ 4) * 256 + at];
                ++tile;
                // (from what lse's rounding and the exponentials explain up to 2^-18 of a logit and 2^-16, far above what a sum has lost; an lse of more classes than these is left alone)
                const float far = fabsf(mass - 1.0f), size = fabsf(mineRow.lse);
                if (far > fmaf(size, 0x1p-24f, 0x1p-21f) && far <= fminf(fmaf(size, 0x1p-18f, 0x1p-16f), 0x1p-10f)) mineRow.weight /= mass;
            }
            for (int k = half; k < pieces; k += 2) {
                Piece o;
                if (!piece_of(t, k, &o)) continue;
                if constexpr (kForm != kLoss) {
                    if (!begin_piece(t, u, k, o)) { ok = false; break; }
                }
                for (int h = 0; h < wide; h += 32) {
                    uint32_t v[32];
                    tmem_load_32cols(tmemBase + buf * 256 + lanes + (uint32_t)(k * wide + h), v);
                    const int c = wide == 64 ? (k - half) + h / 32 : (k - half) / 2;
                    tmem_load_wait();
                    float z[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) z[j] = kInt8 && !p.raw ? (float)(int32_t)v[j] : __uint_as_float(v[j]);      // (raw integers stay what they are)
                    if constexpr (kForm == kLoss) take(z, c, o);
                    else finish(z, mineRow, h, c, o);
                }
                if constexpr (kForm != kLoss) end_piece(t, u, k, o, rowBase);
            }
            if constexpr (kForm == kLoss) {
                const Head &hd = p.head;
                if (!hd.loss) {
                    if (row < p.M) hd.parts[((int64_t)t.n * 2 + half) * p.M + row] = make_float2(terms.top, terms.sum);
                    if (found) hd.picked[row] = picked;
                } else {
                    // One tile takes all classes: the quarter's second warp hands its half to the first, which gives the accumulator back only when it has read it.
                    // So the second is a tile ahead at most, and place and barrier are free again two tiles later.
                    float *const place = reinterpret_cast<float *>(staging) + ((tile & 1) * 4 + q) * 96;
                    if (half) {
                        place[lane] = terms.top;
                        place[32 + lane] = terms.sum;
                        place[64 + lane] = picked;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.handed[q][tile & 1]);
                    } else {
                        if (!warp_wait_for(&sh.handed[q][tile & 1], (tile >> 1) & 1, &sh)) break;
                        join_terms(terms, {place[lane], place[32 + lane]});
                        if (row < p.M) finish_loss(terms, asked.label, hd.classes, found ? picked : place[64 + lane], hd.loss + row, hd.lseOut ? hd.lseOut + row : nullptr, p.status);
                    }
                    ++tile;
                }
            }
            release(buf);
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
template <Form kForm, bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(RCD_PRODUCT_ARGS)
{
    product_body<kForm, kInt8, kAcrossA, kAcrossB, kChunks, false>(mapA, mapB, mapY, mapZ, mapR, p);
}
template <Form kForm, bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) product_pair_kernel(RCD_PRODUCT_ARGS)
{
    product_body<kForm, kInt8, kAcrossA, kAcrossB, kChunks, true>(mapA, mapB, mapY, mapZ, mapR, p);
}
template <Form kForm, bool kInt8, bool kAcrossA, bool kAcrossB, int kChunks>
KernelChoice product_choice(bool pair, int bit)
{
    return pair ? KernelChoice{(const void *)product_pair_kernel<kForm, kInt8, kAcrossA, kAcrossB, kChunks>, bit}
                : KernelChoice{(const void *)product_kernel<kForm, kInt8, kAcrossA, kAcrossB, kChunks>, bit + 1};
}
// By the operands' orders (0: neither across, 1: B, 2: both) and the columns of a piece whose sums are taken in chunks: six kernels each order.
template <Form kForm>
KernelChoice product_choice_by_order(int order, int wide, bool pair, int bit)
{
    auto by_width = [&](auto acrossA, auto acrossB, int at) {
        constexpr bool kA = decltype(acrossA)::value, kB = decltype(acrossB)::value;
        return wide == 0 ? product_choice<kForm, false, kA, kB, 0>(pair, at)
               : wide == 32 ? product_choice<kForm, false, kA, kB, 32>(pair, at + 2) : product_choice<kForm, false, kA, kB, 64>(pair, at + 4);
    };
    const std::false_type along;
    const std::true_type across;
    return order == 0 ? by_width(along, along, bit) : order == 1 ? by_width(along, across, bit + 6) : by_width(across, across, bit + 12);
}

}  // namespace rcd

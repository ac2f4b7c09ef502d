// rcd_orthogonalize of matrices with a side of at most 128: one launch, a cluster of CTAs per matrix, X in shared memory from the first step to the last.
//
// A CTA holds up to 384 columns of X (128 rows, padded with zeros) in slabs of 64, which the tensor cores read either way: along the columns for A = X X^T, across them
// for X = a X + B X.  A needs the sums over all columns: each CTA of the cluster pushes its own to whoever owns the rows, the owners add them up in the
// CTAs' order and push their rows of A to all.  B = b A + c A A and the columns' update are then each CTA's own business.  Nothing but G and the result touches memory,
// and what a step waits for are two exchanges within the cluster where the other forms wait for three barriers over the grid or three launches.
//
// 128 x 128 takes 22 us (all steps in one launch with barriers over the grid: 64), 128 x 2048 51 (82), 16 of 128 x 512 46 (81).  Of the last but one's time a step takes
// 14 000 cycles: the products 4500, the two exchanges with their sums 7000 (latency: 56 KB come and go per CTA), the finishing of B and X the rest.
//
// All threads go through the stages together; thread 0 issues the products.  Every wait is bounded: whoever waits in vain makes its CTA leave, and the others of
// the cluster behind it.
#include "rcd_orthogonal.h"
#include "rcd_tc.cuh"

namespace rcd {

namespace {

constexpr int kSide = 128, kMostThreads = 512, kSlabBytes = kSide * 128, kMostSlabs = 6, kMostCluster = 16;
constexpr int kSquare = 2 * kSlabBytes;                                // A or B: 128 x 128 fp16
constexpr int kExchange = kSide * kSide * 4;
constexpr uint32_t kWaitTurns = 1u << 16;                              // of at most 20 us: a second or so

struct __align__(16) ClusterShared {
    uint64_t product, sums, square;        // a product is complete; the cluster's sums of my rows are here; all of A is
    double squares;                        // of this CTA's columns
    double reduce[kMostThreads / 32];
    uint32_t tmemBase;
    int32_t abort;
};

__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, ClusterShared *sh, uint32_t turns)
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
// All threads: whether all have seen the phase end.
__device__ __forceinline__ bool all_wait_for(uint64_t *bar, uint32_t parity, ClusterShared *sh, uint32_t turns = kWaitTurns)
{
    return __syncthreads_and(wait_for(bar, parity, sh, turns));
}
__device__ __forceinline__ uint32_t cluster_addr(const void *p, int rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    return a;
}
// `bytes` from this CTA's shared memory to another's, reported to its barrier when they are there.
__device__ __forceinline__ void push(uint32_t to, const void *from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" :: "r"(to), "r"(smem_addr(from)), "r"(bytes), "r"(bar) : "memory");
}
// Byte of (row, 16-byte chunk) in a slab of 64 columns, as the 128-byte swizzle places it.
__device__ __forceinline__ int slab_at(int row, int chunk) { return row * 128 + ((chunk ^ (row & 7)) << 4); }
__device__ __forceinline__ uint32_t halves(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 floats(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2 *>(&x)); }
// An operand whose n elements lie next to each other: 16 rows of k are 2048 bytes.
__device__ __forceinline__ uint64_t across_desc(uint32_t addr) { return (make_smem_desc(addr) & ~((uint64_t)0x3fff << 16)) | (uint64_t)(kSlabBytes >> 4) << 16; }
__device__ __forceinline__ void ordered_for_products() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

struct ClusterParams {
    const void *g;
    int64_t ldG, stepG;
    __nv_bfloat16 *o;
    int64_t ldO, stepO;
    int32_t side, len, cluster, slabs, steps;      // slabs per CTA
    bool tall;
    float eps;
    int32_t *status;
    float coefficients[3 * kMostSteps];
};

// Eight neighbours of a row of X, from column col on; zeros outside.
template <typename T, bool kTall, bool kWhole>
__device__ __forceinline__ Pack<T, 8> load_eight(const T *g, int64_t ld, int row, int col, int side, int len)
{
    Pack<T, 8> v;
    if constexpr (kWhole) {
        if (row < side && col < len) return *reinterpret_cast<const Pack<T, 8> *>(g + row * ld + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = from_float<T>(0.0f);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = row < side && col + j < len ? g[kTall ? (int64_t)(col + j) * ld + row : (int64_t)row * ld + col + j] : from_float<T>(0.0f);
    }
    return v;
}

// 512 threads finish the sums of a cluster's CTA sooner (128 x 2048: 51.7 us with them, 53.8 with 256); of CTAs that are alone with a short matrix two go to an SM, if they have 256
// (200 of 128 x 128: 31 us, 46 with 512).
template <bool kAlone> constexpr int kThreadsFor = kAlone ? 256 : kMostThreads;

// kAlone: a cluster of one.  kWhole: rows of a G that is not tall start on 16 bytes and are a multiple of eight long.
template <typename T, bool kTall, bool kWhole, bool kAlone>
__global__ void __launch_bounds__(kThreadsFor<kAlone>, 1) newton_schulz_cluster_kernel(const __grid_constant__ ClusterParams p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int kThreads = kThreadsFor<kAlone>;
    const int slabs = p.slabs, C = kAlone ? 1 : p.cluster, rank = (int)blockIdx.x % C, columns = slabs * 64;
    unsigned char *const x = smem, *const a = x + slabs * kSlabBytes, *const b = a + kSquare;
    float *const exchange = reinterpret_cast<float *>(b + kSquare);
    ClusterShared &sh = *reinterpret_cast<ClusterShared *>(b + kSquare + (C > 1 ? kExchange : 0));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = warp & 3, row = q * 32 + lane;
    constexpr int parts = kThreads / kSide;                            // a warp takes every second part of 32 columns of its 32 rows, or every fourth
    const int part0 = warp >> 2;
    const int64_t matrix = blockIdx.x / C;
    const uint32_t tmemColumns = columns <= 128 ? 256 : 512;           // 128 for the squares, the rest for X

    if (threadIdx.x == 0) {
        mbar_init(&sh.product, 1);
        mbar_init(&sh.sums, 1);
        mbar_init(&sh.square, 1);
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_addr(&sh.tmemBase)), "r"(tmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // The launch behind this one may begin when all CTAs have their tensor memory: it may ask for all of it, and keeps it while it waits for this one's end.
    __syncthreads();
    after_the_one_before();

    // The norm: each CTA's columns, then the cluster's in their order.
    const T *const g = (const T *)p.g + matrix * p.stepG;
    const int first = rank * columns, pieces = kSide * columns / 8;
    auto place = [&](int i, int *r, int *c) {                          // (neighbouring threads along G's rows)
        if (kTall) { *r = i % kSide; *c = i / kSide * 8; }
        else { *r = i / (columns / 8); *c = i % (columns / 8) * 8; }
    };
    // (16-bit elements wait in their place in shared memory until the norm is known; fp32 is read again.  In registers, with the loops unrolled, the code itself took 9000 cycles to come.)
    auto at_piece = [&](int r, int c) { return x + c / 64 * kSlabBytes + slab_at(r, c % 64 / 8); };
    double s = 0.0;
#pragma unroll (kWhole ? 4 : 1)
    for (int i = threadIdx.x; i < pieces; i += kThreads) {
        int r, c;
        place(i, &r, &c);
        const Pack<T, 8> v = load_eight<T, kTall, kWhole>(g, p.ldG, r, first + c, p.side, p.len);
        if constexpr (sizeof(T) == 2) *reinterpret_cast<Pack<T, 8> *>(at_piece(r, c)) = v;
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fma((double)to_float(v.v[j]), (double)to_float(v.v[j]), s);
    }
    s = warp_sum(s);
    if (lane == 0) sh.reduce[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kThreads / 32; ++i) s += sh.reduce[i];
        sh.squares = s;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                                                 // all are here: barriers and sums exist
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh.tmemBase, lanes = (uint32_t)(q * 32) << 16;
    double all = 0.0;
    for (int k = 0; k < C; ++k) {
        double part;
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(part) : "r"(cluster_addr(&sh.squares, k)) : "memory");
        all += part;
    }
    const double norm = sqrt(all) + (double)p.eps;
    int e = 0;
    float factor = norm == 0.0 ? 0.0f : NAN;                           // (of nothing: zeros; a G that is not finite: NaN)
    if (norm > 0.0 && norm < (double)INFINITY) {
        e = kUp - 1 - ilogb(norm);
        factor = (float)(ldexp(1.0, kUp) / ldexp(norm, e));
    }
    const float up0 = ldexpf(1.0f, e / 2), up1 = ldexpf(1.0f, e - e / 2);          // (2^e alone may be out of fp32's range)
#pragma unroll (kWhole || sizeof(T) == 2 ? 4 : 1)
    for (int i = threadIdx.x; i < pieces; i += kThreads) {
        int r, c;
        place(i, &r, &c);
        Pack<T, 8> v;
        if constexpr (sizeof(T) == 2) v = *reinterpret_cast<const Pack<T, 8> *>(at_piece(r, c));
        else v = load_eight<T, kTall, kWhole>(g, p.ldG, r, first + c, p.side, p.len);
        auto z = [&](int j) { return to_float(v.v[j]) * up0 * up1; };
        *reinterpret_cast<uint4 *>(at_piece(r, c)) = make_uint4(halves(z(0), z(1)), halves(z(2), z(3)), halves(z(4), z(5)), halves(z(6), z(7)));
    }
    ordered_for_products();
    __syncthreads();

    constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(kSide >> 4) << 24);        // fp16 x fp16 -> fp32, 128 rows
    const uint32_t xAt = smem_addr(x), aAt = smem_addr(a), bAt = smem_addr(b);
    const float down = 1.0f / (1 << kUp);
    const int owned = kSide / C;                                       // rows of A that this CTA adds up
    uint32_t products = 0;
    // thread 0 has issued a product: all wait for it
    auto complete = [&] { return all_wait_for(&sh.product, products++ & 1, &sh); };
    // 32 columns of the thread's row, from tensor memory on
    auto sums_of = [&](uint32_t column, uint32_t (&v)[32]) {
        tmem_load_32cols(tmem + lanes + column, v);
        tmem_load_wait();
    };
    // Before the next product writes where others have read.
    auto handed_over = [&] {
        ordered_for_products();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    // 128 rows of 128 bytes: the slabs of A, then of B
    auto quarter = [&](int k) { return a + k * kSlabBytes; };
    bool ok = true;
    for (int i = 0; i < p.steps; ++i) {
        const float *const c = p.coefficients + 3 * i;
        const float f = i == 0 ? factor : 1.0f;
        // ---- A = X X^T ----
        if (threadIdx.x == 0) {
            for (int k = 0; k < 4 * slabs; ++k) {
                const uint64_t d = make_smem_desc(xAt + (uint32_t)(k / 4 * kSlabBytes)) + 2 * (k % 4);
                mma_issue<false>(tmem, d, d, kIdesc | ((uint32_t)(kSide >> 3) << 17), k > 0);
            }
            mma_commit(&sh.product);
            if (C > 1) {
                mbar_expect_tx(&sh.sums, kExchange - owned * 512);     // (but for what comes from here)
                mbar_expect_tx(&sh.square, kSquare - owned * 256);     // (but for my own rows)
            }
        }
        if (!(ok = complete())) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float alpha = down * (f * f);
#pragma unroll
        for (int h = 0; h < 4 / parts; ++h) {
            const int part = part0 + h * parts;
            uint32_t v[32];
            sums_of((uint32_t)(part * 32), v);
            if (C == 1) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    auto z = [&](int j) { return __uint_as_float(v[8 * k + j]) * alpha; };
                    *reinterpret_cast<uint4 *>(a + part / 2 * kSlabBytes + slab_at(row, part % 2 * 4 + k)) = make_uint4(halves(z(0), z(1)), halves(z(2), z(3)), halves(z(4), z(5)), halves(z(6), z(7)));
                }
            } else {
                // a row's 128 sums are four times 128 bytes: those of my own rows where they are added up, the others' in the places of that row of A and B
                unsigned char *const to = row / owned == rank ? (unsigned char *)exchange + ((rank * 4 + part) * owned + row % owned) * 128 : quarter(part) + row * 128;
#pragma unroll
                for (int k = 0; k < 8; ++k) *reinterpret_cast<uint4 *>(to + ((k ^ (row & 7)) << 4)) = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
            }
        }
        if (C > 1) {
            // To the rows' owners.  (What an owner sends back comes into the place that its sums were read from; my own rows of A, which the others may still be waiting for, are
            // written next when all have sent sums of the next step, and so have had them.)
            ordered_for_products();
            __syncthreads();
            if (threadIdx.x < 4 * C && (int)threadIdx.x / 4 != rank) {
                const int owner = threadIdx.x / 4, piece = threadIdx.x % 4;
                push(cluster_addr(exchange + (rank * 4 + piece) * owned * 32, owner), quarter(piece) + owner * owned * 128, (uint32_t)owned * 128, cluster_addr(&sh.sums, owner));
            }
            if (!(ok = all_wait_for(&sh.sums, i & 1, &sh))) break;
            // four columns at a time, 32 pieces of a row
            for (int piece = threadIdx.x; piece < owned * 32; piece += kThreads) {
                const int r = piece / 32, mine = rank * owned + r, col = piece % 32 * 4;
                float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
                for (int k = 0; k < C; ++k) {
                    const float4 from = *reinterpret_cast<const float4 *>(exchange + ((k * 4 + col / 32) * owned + r) * 32 + (((col % 32 / 4) ^ (mine & 7)) << 2));
                    z.x += from.x; z.y += from.y; z.z += from.z; z.w += from.w;
                }
                *reinterpret_cast<uint2 *>(a + col / 64 * kSlabBytes + slab_at(mine, col % 64 / 8) + col % 8 * 2) = make_uint2(halves(z.x * alpha, z.y * alpha), halves(z.z * alpha, z.w * alpha));
            }
            ordered_for_products();
            __syncthreads();
            if (threadIdx.x < 2 * C && (int)threadIdx.x / 2 != rank) {
                unsigned char *const at = a + threadIdx.x % 2 * kSlabBytes + rank * owned * 128;
                push(cluster_addr(at, threadIdx.x / 2), at, (uint32_t)owned * 128, cluster_addr(&sh.square, threadIdx.x / 2));
            }
            if (!(ok = all_wait_for(&sh.square, i & 1, &sh))) break;
        }
        handed_over();
        // ---- B = b A + c A A ----
        if (threadIdx.x == 0) {
            for (int k = 0; k < 8; ++k) {
                const uint64_t d = make_smem_desc(aAt + (uint32_t)(k / 4 * kSlabBytes)) + 2 * (k % 4);
                mma_issue<false>(tmem, d, d, kIdesc | ((uint32_t)(kSide >> 3) << 17), k > 0);
            }
            mma_commit(&sh.product);
        }
        if (!(ok = complete())) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float polyAlpha = c[2] * down, polyBeta = c[1];
#pragma unroll
        for (int h = 0; h < 4 / parts; ++h) {
            const int part = part0 + h * parts;
            uint32_t v[32];
            sums_of((uint32_t)(part * 32), v);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = part / 2 * kSlabBytes + slab_at(row, part % 2 * 4 + k);
                const uint4 old = *reinterpret_cast<const uint4 *>(a + at);
                const uint32_t w[4] = {old.x, old.y, old.z, old.w};
                uint32_t z[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 r = floats(w[j]);
                    z[j] = halves(fmaf(polyBeta, r.x, __uint_as_float(v[8 * k + 2 * j]) * polyAlpha), fmaf(polyBeta, r.y, __uint_as_float(v[8 * k + 2 * j + 1]) * polyAlpha));
                }
                *reinterpret_cast<uint4 *>(b + at) = make_uint4(z[0], z[1], z[2], z[3]);
            }
        }
        handed_over();
        // ---- X = a X + B X ----
        if (threadIdx.x == 0) {
            for (int n = 0; n < slabs; ++n)
                for (int k = 0; k < 8; ++k)
                    mma_issue<false>(tmem + kSide + 64 * n, make_smem_desc(bAt + (uint32_t)(k / 4 * kSlabBytes)) + 2 * (k % 4), across_desc(xAt + (uint32_t)(n * kSlabBytes)) + 128 * k,
                                     kIdesc | (1u << 16) | ((uint32_t)(64 >> 3) << 17), k > 0);
            mma_commit(&sh.product);
        }
        if (!(ok = complete())) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const bool last = i == p.steps - 1;
        const float xAlpha = (last ? down * down : down) * f, xBeta = (last ? down : 1.0f) * c[0] * f;
        for (int part = part0; part < 2 * slabs; part += parts) {
            const int n = part / 2, half = part % 2;
            uint32_t v[32];
            sums_of((uint32_t)(kSide + 64 * n + half * 32), v);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint4 *const at = reinterpret_cast<uint4 *>(x + n * kSlabBytes + slab_at(row, 4 * half + k));
                const uint4 old = *at;
                const uint32_t w[4] = {old.x, old.y, old.z, old.w};
                float z[8];
                [[maybe_unused]] Pack<T, 8> whole;                     // (an fp32 G itself in the first step's sum: fp16 leaves 11 bits of it)
                if constexpr (sizeof(T) == 4) {
                    if (i == 0) whole = load_eight<T, kTall, kWhole>(g, p.ldG, row, first + 64 * n + half * 32 + 8 * k, p.side, p.len);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float2 r = floats(w[j]);
                    if constexpr (sizeof(T) == 4) {
                        if (i == 0) r = make_float2(whole.v[2 * j] * up0 * up1, whole.v[2 * j + 1] * up0 * up1);
                    }
                    z[2 * j] = fmaf(xBeta, r.x, __uint_as_float(v[8 * k + 2 * j]) * xAlpha);
                    z[2 * j + 1] = fmaf(xBeta, r.y, __uint_as_float(v[8 * k + 2 * j + 1]) * xAlpha);
                }
                if (!last) {
                    *at = make_uint4(halves(z[0], z[1]), halves(z[2], z[3]), halves(z[4], z[5]), halves(z[6], z[7]));
                } else if (row < p.side) {
                    const int col = first + 64 * n + half * 32 + 8 * k;
                    __nv_bfloat16 *const o = p.o + matrix * p.stepO + (kTall ? (int64_t)col * p.ldO + row : (int64_t)row * p.ldO + col);
                    if (!kTall && col + 8 <= p.len && ((uintptr_t)o) % 16 == 0) store_pack<8>(o, z);
                    else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (col + j < p.len) o[kTall ? j * p.ldO : j] = __float2bfloat16_rn(z[j]);
                    }
                }
            }
        }
        if (!last) handed_over();
    }
    if (!ok) let_copies_land();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();                                                 // nothing of the others is on its way here any more
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(tmemColumns) : "memory");
    }
    if (threadIdx.x == 0 && !ok) atomicOr(p.status, kDevTimeout);
}

// A cluster's waits for sums that nobody sends: the first has to run out for every thread, and the one behind it to be given up at once.
__global__ void __launch_bounds__(64) cluster_wait_selftest_kernel(int32_t *status)
{
    __shared__ ClusterShared sh;
    if (threadIdx.x == 0) {
        mbar_init(&sh.sums, 1);
        mbar_init(&sh.square, 1);
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const bool came = all_wait_for(&sh.sums, 0, &sh, 1u << 5);
    const bool then = all_wait_for(&sh.square, 0, &sh);
    if (threadIdx.x == 0) atomicOr(status, came || then || !sh.abort ? kDevBadState : kDevTimeout);
}

int shared_bytes(int cluster, int slabs) { return slabs * kSlabBytes + 2 * kSquare + (cluster > 1 ? kExchange : 0) + (int)sizeof(ClusterShared); }

typedef void (*ClusterKernel)(ClusterParams);
template <typename T, bool kAlone>
ClusterKernel kernel_for(bool tall, bool whole)
{
    return tall ? newton_schulz_cluster_kernel<T, true, false, kAlone> : whole ? newton_schulz_cluster_kernel<T, false, true, kAlone> : newton_schulz_cluster_kernel<T, false, false, kAlone>;
}
template <typename T>
ClusterKernel kernel_for(bool alone, bool tall, bool whole) { return alone ? kernel_for<T, true>(tall, whole) : kernel_for<T, false>(tall, whole); }

}  // namespace

rcd_status launch_cluster_wait_selftest(rcd_ctx *ctx, int32_t *status, cudaStream_t st)
{
    cluster_wait_selftest_kernel<<<1, 64, 0, st>>>(status);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

// Whether the device takes a cluster of 16 that fill an SM each.
static bool sixteen(rcd_ctx *ctx)
{
    if (ctx->clusterSixteen < 0) {
        ctx->clusterSixteen = 0;
        auto *kernel = newton_schulz_cluster_kernel<float, true, false, false>;
        const int bytes = shared_bytes(kMostCluster, kMostSlabs);
        int n = 0;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = kMostCluster;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t config{};
        config.gridDim = dim3(kMostCluster);
        config.blockDim = dim3(kMostThreads);
        config.dynamicSmemBytes = (size_t)bytes;
        config.attrs = &attr;
        config.numAttrs = 1;
        if (cudaSetDevice(ctx->device) == cudaSuccess && allow_shared(kernel, bytes) == cudaSuccess && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
            cudaOccupancyMaxActiveClusters(&n, kernel, &config) == cudaSuccess)
            ctx->clusterSixteen = n > 0;
        else
            cudaGetLastError();
    }
    return ctx->clusterSixteen != 0;
}

// The smallest cluster whose CTAs hold X, of up to four slabs each, or six where it is eight or sixteen of them.
int cluster_for(rcd_ctx *ctx, int64_t rows, int64_t cols)
{
    const int64_t side = std::min(rows, cols), slabs = (std::max(rows, cols) + 63) / 64;
    if (side > kSide) return 0;
    for (int c = 1; c <= kMostCluster; c *= 2)
        if (slabs <= c * (c < 8 ? 4 : kMostSlabs)) return c < 16 || sixteen(ctx) ? c : 0;
    return 0;
}

rcd_status launch_cluster(rcd_ctx *ctx, const rcd_orthogonalize_args &a, int cluster, cudaStream_t st)
{
    ClusterParams p{};
    p.g = a.g_dev;
    p.ldG = a.ld_g;
    p.stepG = a.batch > 1 ? a.step_g : 0;
    p.o = (__nv_bfloat16 *)a.o_dev;
    p.ldO = a.ld_o;
    p.stepO = a.batch > 1 ? a.step_o : 0;
    p.tall = a.rows > a.cols;
    p.side = (int32_t)std::min(a.rows, a.cols);
    p.len = (int32_t)std::max(a.rows, a.cols);
    p.cluster = cluster;
    p.slabs = (int32_t)(((p.len + 63) / 64 + cluster - 1) / cluster);
    p.steps = a.steps;
    p.eps = a.eps;
    p.status = ctx->statusOwn + kOperatorStatus;
    for (int i = 0; i < 3 * a.steps; ++i) p.coefficients[i] = a.coefficients_host[i];
    const int64_t eb = elem_bytes(a.type);
    const bool whole = rows_aligned(a.g_dev, a.ld_g, eb, 16) && a.cols % 8 == 0 && (a.batch == 1 || a.step_g * eb % 16 == 0);
    const bool alone = cluster == 1;
    const ClusterKernel kernel = a.type == RCD_ELEM_BF16 ? kernel_for<__nv_bfloat16>(alone, p.tall, whole) : a.type == RCD_ELEM_F16 ? kernel_for<__half>(alone, p.tall, whole)
                                                                                                                          : kernel_for<float>(alone, p.tall, whole);
    const int bit = 3 * (a.type == RCD_ELEM_BF16 ? 0 : a.type == RCD_ELEM_F16 ? 1 : 2) + (p.tall ? 0 : whole ? 1 : 2) + (alone ? 9 : 0);
    if (!(ctx->clusterReady >> bit & 1)) {
        RCD_CUDA(ctx, allow_shared(kernel, shared_bytes(2, kMostSlabs)));
        RCD_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        ctx->clusterReady |= 1u << bit;
    }
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = (unsigned)cluster;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)(a.batch * cluster));
    config.blockDim = dim3(alone ? kThreadsFor<true> : kThreadsFor<false>);
    config.dynamicSmemBytes = (size_t)shared_bytes(cluster, p.slabs);
    config.stream = st;
    config.attrs = attrs;
    config.numAttrs = 2;
    ctx->kernelLaunches++;
    ctx->tcLaunches++;
    RCD_CUDA(ctx, cudaLaunchKernelEx(&config, kernel, p));
    return RCD_OK;
}

}  // namespace rcd

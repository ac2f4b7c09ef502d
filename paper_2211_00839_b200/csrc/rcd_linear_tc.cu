// Matrix products of rcd_linear and its gradients on the tensor cores (rcd_product.cuh): which tile, the launches, the join of
// pieces of the k axis.
#include "rcd_norm.cuh"
#include "rcd_product.cuh"

namespace rcd {

namespace {

// Joins the pieces of the k axis in their order, then the epilogue: four columns per thread.
template <bool kInt8>
__global__ void __launch_bounds__(256) join_kernel(const void *__restrict__ parts, int32_t splits, int32_t M, int64_t rowsPart, int32_t N, int64_t ld, const __grid_constant__ Epilogue e,
                                                   const __grid_constant__ Scaling sc)
{
    after_the_one_before();
    const int perRow = (N + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)M * perRow) return;
    const int64_t m = i / perRow;
    const int n = (int)(i - m * perRow) * 4;
    float z[4];
    if constexpr (kInt8) {
        int4 s = make_int4(0, 0, 0, 0);
#pragma unroll 8
        for (int k = 0; k < splits; ++k) {
            const int4 x = __ldcs((const int4 *)((const int32_t *)parts + (k * rowsPart + m) * ld + n));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        z[0] = (float)s.x; z[1] = (float)s.y; z[2] = (float)s.z; z[3] = (float)s.w;
    } else {
        float4 s = make_float4(0, 0, 0, 0);
#pragma unroll 8
        for (int k = 0; k < splits; ++k) {
            const float4 x = __ldcs((const float4 *)((const float *)parts + (k * rowsPart + m) * ld + n));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        z[0] = s.x; z[1] = s.y; z[2] = s.z; z[3] = s.w;
    }
    const float sx = e.xs ? e.xs[m] : sc.alpha * (sc.factor ? sc.alphaPower == 1 ? *sc.factor : sc.alphaPower == 2 ? *sc.factor * *sc.factor : 1.0f : 1.0f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (n + j >= N) break;
        z[j] *= sx;
        if (e.ws) z[j] *= e.ws[n + j];
        if (e.bias) z[j] += e.bias[n + j];
    }
    auto whole = [&](const void *base, int64_t ld2, rcd_elem type) {
        const int64_t eb = type == RCD_ELEM_F32 ? 4 : 2;
        return n + 4 <= N && (((uintptr_t)base + (uintptr_t)((m * ld2 + n) * eb)) % (4 * eb)) == 0;
    };
    auto put = [&](void *base, int64_t ld2, const float (&v)[4]) {
        if (whole(base, ld2, e.type)) store_typed<4>(base, m * ld2 + n, e.type, v);
        else
            for (int j = 0; j < 4 && n + j < N; ++j) { const float o[1] = {v[j]}; store_typed<1>(base, m * ld2 + n + j, e.type, o); }
    };
    if (e.z) put(e.z, e.ldz, z);
    activate(z, e.act);
    const float f = sc.factor ? *sc.factor : 1.0f, beta = sc.beta * (sc.betaPower == 0 ? 1.0f : sc.betaPower == 1 ? f : f * f);
    if (e.residual) {
        float r[4] = {0, 0, 0, 0};
        // (its type may be another: an update's last product adds fp16 to what leaves as bf16)
        if (whole(e.residual, e.ldr, sc.residualType)) load_typed<4>(r, e.residual, m * e.ldr + n, sc.residualType);
        else
            for (int j = 0; j < 4 && n + j < N; ++j) { float o[1]; load_typed<1>(o, e.residual, m * e.ldr + n + j, sc.residualType); r[j] = o[0]; }
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = fmaf(beta, r[j], z[j]);
        if (sc.low) {                                      // (rows of whole 64s)
            load_pack<4>(r, (const __half *)sc.low + m * e.ldr + n);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = fmaf(beta * (1.0f / (1 << kLowUp)), r[j], z[j]);
        }
    }
    put(e.y, e.ldy, z);
}

// Rows of any start and distance to rows that start on 16 bytes: 16 bytes per thread.
template <typename T>
__global__ void __launch_bounds__(256) pack_kernel(const T *__restrict__ src, int64_t ld, int64_t rows, int64_t len, T *__restrict__ dst, int64_t ldDst)
{
    after_the_one_before();
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
    __shared__ ProductShared sh;
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
    int tn, splits, slabsPerSplit, band, subM, subN;
    double cycles;                                       // an estimate
    int64_t slabs, tilesM, tilesN, tiles, rowsPart, ldPart;     // rowsPart: whole pieces of 32 rows, which are stored whole
    bool packA, packB;
    int64_t ldA, ldB;
    size_t partAt, aAt, bAt, bytes;
};


// Slabs of a tile from which on its warps have one place for their pieces: gradients of 8192 x 4096 x 4096 (64 and 128 slabs) 419 us for 438; from 16 on the int8 product of
// 50 000 x 2048 x 2048 with its residual would take 193 us for 180.
constexpr int kOnePlaceFrom = 48;
// Column tiles that are neighbours in the order of the work, where B has more bytes than stay in L2.  (8192 x 4096 x 65 536: 3.36 ms, 4.25 row after row;
// all gradients over 32 768 classes 5.10 ms and 5.64.)
constexpr int kBand = 8;
constexpr int64_t kBandFrom = 48LL << 20;

// Which tile, and into how many pieces the k axis is cut: the least of an estimate in cycles.  A slab costs an SM its share of the
// tensor pipe (128 x 256 x 128 bytes: 512 cycles) or what its operands take from L2 (some 56 bytes a cycle), a tile its epilogue behind the
// last slab; pieces cost the join's launch and their way through L2.  A head's products are not cut along k (exponentials want whole logits), nor are symmetric ones and batches; a head's
// epilogue, some 12 cycles a column, can take longer than the slabs of a tile.  Symmetric products take the tiles of the square blocks on
// and below the diagonal.
Plan make_plan(const rcd_ctx *ctx, const Product &p, bool packA, bool packB)
{
    Plan best{};
    const int64_t eb = elem_bytes(p.type);
    best.packA = packA;
    best.packB = packB;
    const int64_t slabElems = kSlab / eb;
    const int64_t slabs = (p.K + slabElems - 1) / slabElems;
    const bool head = p.form == kLoss || p.form == kLogitGrads, whole = head || p.symmetric || p.batch > 1;
    const int64_t batch = std::max<int64_t>(p.batch, 1);
    double least = 1e300;
    for (int pair = 0; pair < 2; ++pair)
        for (int tn = 64; tn <= 256; tn += p.form == kLoss && !pair ? 32 : 64) {       // (rounds of 64 columns where whole pieces of 16-bit output are stored)
            if (pair && p.b.across && tn % 128 != 0) continue;         // (boxes of 64 columns per CTA)
            if (pair && ctx->smCount < 2) continue;
            if (p.oneTile && tn < p.N) continue;
            const int64_t tilesM = (p.M + (pair ? 256 : 128) - 1) / (pair ? 256 : 128), tilesN = (p.N + tn - 1) / tn;
            const int64_t slots = pair ? ctx->smCount / 2 : ctx->smCount;
            int64_t tiles = tilesM * tilesN;
            const int rowsTile = pair ? 256 : 128, block = std::max(rowsTile, tn);
            if (p.symmetric) {
                if (block % rowsTile || block % tn) continue;
                const int64_t blocks = (p.M + block - 1) / block;
                tiles = blocks * (blocks + 1) / 2 * (block / rowsTile) * (block / tn);
            }
            if (tiles * batch > 0x3fffffffLL) continue;
            const double aRows = head && !pair ? (double)std::min<int64_t>(p.M, 128) : 128.0;
            const double slab = std::max(512.0 * tn / 256.0, (aRows + (pair ? tn / 2 : tn)) * kSlab / 56.0) + 10.0;
            for (int splits = 1; splits <= 64; ++splits) {
                if (splits > 1 && (whole || tiles * splits > 2 * slots || splits > slabs)) break;
                const int64_t per = (slabs + splits - 1) / splits;
                if (splits > 1 && (splits - 1) * per >= slabs) continue;     // (an empty piece)
                const int64_t waves = (tiles * batch * splits + slots - 1) / slots;
                double t = (double)waves * std::max((double)per * slab, head ? 12.0 * tn : 0.0) + 2500.0 + 9.0 * tn;
                if (splits > 1) t += 6000.0 + (double)p.M * (double)p.N * 8.0 * splits / 5000.0;
                if (t < least) {
                    least = best.cycles = t;
                    best.pair = pair != 0;
                    best.tn = tn;
                    best.splits = splits;
                    best.slabsPerSplit = (int)per;
                    best.slabs = slabs;
                    best.tilesM = tilesM;
                    best.tilesN = tilesN;
                    best.tiles = tiles;
                    best.subM = p.symmetric ? block / rowsTile : 0;
                    best.subN = p.symmetric ? block / tn : 0;
                }
            }
        }
    // Rows of tiles one after the other read all of B again and again: from L2, as long as it fits there.
    best.band = (int)best.tilesN;
    if (!p.symmetric && p.N * p.K * eb > kBandFrom) best.band = std::min(best.band, kBand);
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

// A call asks three times (workspace twice, launch), a program the same sizes over and over: the last sixteen answers are kept, by
// sizes, types and orders alone.
struct PlanCache {
    struct Entry { int64_t M, N, K, ldA, ldB, batch; int how; Plan plan; } of[16];
    unsigned next;
};
const Plan &plan_product(rcd_ctx *ctx, const Product &p)
{
    static_assert(sizeof(PlanCache) <= sizeof(ctx->productPlans) && std::is_trivially_copyable<PlanCache>::value, "the context has room for it");
    PlanCache &c = *reinterpret_cast<PlanCache *>(ctx->productPlans);      // (zeros at first: how 0 is nobody's)
    const int64_t eb = elem_bytes(p.type);
    const bool packA = !rows_mappable(p.a.p, p.a.ld, eb), packB = !rows_mappable(p.b.p, p.b.ld, eb);
    const int how = 1 | (int)p.type << 1 | (int)p.a.across << 3 | (int)p.b.across << 4 | (int)packA << 5 | (int)packB << 6 | (int)p.form << 7 | (int)p.symmetric << 9 | (int)p.oneTile << 10;
    for (const PlanCache::Entry &e : c.of)
        if (e.how == how && e.M == p.M && e.N == p.N && e.K == p.K && e.ldA == p.a.ld && e.ldB == p.b.ld && e.batch == p.batch) return e.plan;
    PlanCache::Entry &e = c.of[c.next++ % 16];
    e = {p.M, p.N, p.K, p.a.ld, p.b.ld, p.batch, how, make_plan(ctx, p, packA, packB)};
    return e.plan;
}

rcd_status encode(rcd_ctx *ctx, CUtensorMap *map, CUtensorMapDataType type, const void *p, int64_t inner, int64_t outer, int64_t ldBytes, int boxInner, int boxOuter,
                  CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(ctx, RCD_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
    const cuuint64_t strides[1] = {(cuuint64_t)ldBytes};
    const cuuint32_t box[2] = {(cuuint32_t)boxInner, (cuuint32_t)boxOuter};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult cr = fn(map, type, 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (cr != CUDA_SUCCESS) return fail(ctx, RCD_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d", (int)cr);
    return RCD_OK;
}
CUtensorMapDataType map_type(rcd_elem t)
{
    return t == RCD_ELEM_I8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : t == RCD_ELEM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
           : t == RCD_ELEM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
}

KernelChoice plain_kernel(bool i8, int order, int wide, bool pair)
{
    return i8 ? product_choice<kPlain, true, false, false, 0>(pair, 0) : product_choice_by_order<kPlain>(order, wide, pair, 2);
}

rcd_status run_product(rcd_ctx *ctx, const KernelChoice &c, int grid, size_t smem, CUtensorMap (&maps)[5], TcParams &q, cudaStream_t st)
{
    if (!(ctx->productReady >> c.bit & 1)) {            // (shared memory beyond 48 KB is asked for once per context and kernel)
        cudaFuncAttributes at;
        RCD_CUDA(ctx, cudaFuncGetAttributes(&at, c.kernel));
        if (at.numRegs < kLaunchRegs) return fail(ctx, RCD_ERR_INTERNAL, "a product's kernel has %d registers a thread, too few for its warpgroups' split", at.numRegs);
        RCD_CUDA(ctx, cudaFuncSetAttribute(c.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared));
        ctx->productReady |= 1ull << c.bit;
    }
    void *args[6] = {&maps[0], &maps[1], &maps[2], &maps[3], &maps[4], &q};
    // The launch may overtake the end of the kernel before it: barriers, tensor memory and maps are ready by then, and griddepcontrol.wait comes before the first
    // access to memory.
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)grid);
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = smem;
    config.stream = st;
    config.attrs = &early;
    config.numAttrs = 1;
    ctx->kernelLaunches++;
    ctx->tcLaunches++;
    RCD_CUDA(ctx, cudaLaunchKernelExC(&config, c.kernel, args));
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

int64_t product_tile_columns(rcd_ctx *ctx, const Product &p) { return plan_product(ctx, p).tilesN; }
double product_cycles(rcd_ctx *ctx, const Product &p) { return plan_product(ctx, p).cycles; }

bool rows_mappable(const void *p, int64_t ld, int64_t eb) { return ((uintptr_t)p) % 16 == 0 && ld * eb % 16 == 0 && ld * eb < (1LL << 40); }

rcd_status launch_pack(rcd_ctx *ctx, const void *from, int64_t ld, int64_t rows, int64_t len, int64_t eb, void *to, int64_t ldTo, cudaStream_t st)
{
    const dim3 grid((unsigned)std::min<int64_t>((rows * (ldTo * eb / 16) + 255) / 256, (int64_t)ctx->smCount * 16));
    return eb == 1 ? launch_early(ctx, pack_kernel<int8_t>, grid, 256, st, (const int8_t *)from, ld, rows, len, (int8_t *)to, ldTo)
                   : launch_early(ctx, pack_kernel<uint16_t>, grid, 256, st, (const uint16_t *)from, ld, rows, len, (uint16_t *)to, ldTo);
}

size_t product_workspace(rcd_ctx *ctx, const Product &p) { return p.form == kPlain && few_rows(p) ? 0 : plan_product(ctx, p).bytes; }

rcd_status launch_product(rcd_ctx *ctx, const Product &p, void *workspace, cudaStream_t st)
{
    if (p.form == kPlain && few_rows(p)) return launch_few_rows(ctx, p, st);
    const Plan plan = plan_product(ctx, p);
    unsigned char *ws = (unsigned char *)workspace;
    const int64_t eb = elem_bytes(p.type);
    const bool i8 = p.type == RCD_ELEM_I8;
    const int64_t batch = std::max<int64_t>(p.batch, 1);
    if (batch > 1 && (plan.packA || plan.packB)) return fail(ctx, RCD_ERR_INTERNAL, "a batch's operands start on 16 bytes");
    auto operand = [&](const Operand &o, int64_t mn, bool pack, int64_t ld, size_t at, int boxRows, int64_t step, CUtensorMap *map) {
        const int64_t rows = (batch - 1) * step + (o.across ? p.K : mn), len = o.across ? mn : p.K;
        const void *from = o.p;
        if (pack) {
            RCD_TRY(launch_pack(ctx, o.p, o.ld, rows, len, eb, ws + at, ld, st));
            from = ws + at;
        }
        return encode(ctx, map, map_type(p.type), from, len, rows, ld * eb, o.across ? 64 : (int)(kSlab / eb), o.across ? kSlabRows16 : boxRows);
    };
    // (few rows take no place for 128: what the instruction reads behind them are rows that nobody looks at)
    const int aRows = p.a.across || plan.pair ? kRows : (int)std::min<int64_t>(kRows, (p.M + 7) / 8 * 8);
    CUtensorMap maps[5] = {};
    RCD_TRY(operand(p.a, p.M, plan.packA, plan.ldA, plan.aAt, aRows, p.aStep, &maps[0]));
    RCD_TRY(operand(p.b, p.N, plan.packB, plan.ldB, plan.bAt, plan.pair ? plan.tn / 2 : plan.tn, p.bStep, &maps[1]));

    TcParams q{};
    q.M = (int32_t)p.M; q.N = (int32_t)p.N;
    q.walk = {(int32_t)plan.tilesM, (int32_t)plan.tilesN, (int32_t)plan.tiles, plan.band, plan.splits, plan.subM, plan.subN};
    q.units = (int32_t)(plan.tiles * plan.splits * batch);
    q.aStep = (int32_t)p.aStep; q.bStep = (int32_t)p.bStep; q.yStep = (int32_t)p.yStep; q.rStep = (int32_t)p.rStep;
    q.head = p.head;
    q.s = p.scaling;
    q.slabs = (int32_t)plan.slabs;
    q.slabsPerSplit = plan.slabsPerSplit;
    q.tn = plan.tn;
    const int chunk = p.oneTile || p.out.type == RCD_ELEM_F32 ? kChunkSlabs : p.head.sums ? kChunkSlabsSums : kChunkSlabs16;
    const bool chunks = !i8 && plan.slabsPerSplit > (chunk == kChunkSlabs16 ? 2 * chunk : chunk);
    q.chunk = chunks ? chunk : q.slabs;
    q.aRows = aRows;
    q.e = p.out;
    q.raw = plan.splits > 1;
    // What the ring leaves room for.  A second place per warp hides a store's way out behind the next piece, which does not matter where a tile's slabs take longer than
    // its end; with one, and without columns, 256 x 256 tiles have a ring of six stages for four.
    q.columnBytes = !q.raw && (q.e.bias || (i8 && q.e.ws) || p.oneTile) ? kColumnBytes : 0;
    q.places = !q.raw && (q.e.z || p.symmetric || p.head.sums) ? 2 : plan.slabsPerSplit >= kOnePlaceFrom ? 1 : 2;
    q.stagingBytes = p.form == kLoss ? kJoinStaging : kEpiWarps * q.places * kPiece;
    const OperandRing ring = ring_of(q.aRows, plan.pair ? plan.tn / 2 : plan.tn, q.stagingBytes + q.columnBytes + kFixedShared);
    q.stageBytes = ring.stageBytes;
    q.stages = ring.stages;
    q.idesc = (i8 ? (2u << 4) | (1u << 7) | (1u << 10)                                     // S8 x S8 -> S32
                  : (1u << 4) | (p.type == RCD_ELEM_BF16 ? (1u << 7) | (1u << 10) : 0u)) | // BF16 x BF16 or F16 x F16 -> F32
              (p.a.across ? 1u << 15 : 0u) | (p.b.across ? 1u << 16 : 0u) | ((uint32_t)(plan.tn >> 3) << 17) | ((uint32_t)((plan.pair ? 256 : 128) >> 4) << 24);
    if (q.raw) {
        q.e = Epilogue{};
        q.e.type = RCD_ELEM_F32;
        q.e.y = ws + plan.partAt;
        q.e.ldy = plan.ldPart;
        q.rowsPart = (int32_t)plan.rowsPart;
    }
    q.status = ctx->statusOwn + kOperatorStatus;
    const int64_t yb = elem_bytes(q.e.type);
    auto rows_of = [&](int64_t step) { return q.raw ? plan.splits * plan.rowsPart : (batch - 1) * step + p.M; };
    auto output = [&](const void *base, int64_t ld, rcd_elem type, int64_t step, bool *use, CUtensorMap *map) {
        *use = base && rows_aligned(base, ld, yb, 16) && ld * yb < (1LL << 40);
        return *use ? encode(ctx, map, map_type(type), base, q.raw ? plan.ldPart : p.N, rows_of(step), ld * yb, (int)(128 / yb), 32) : RCD_OK;
    };
    RCD_TRY(output(q.e.y, q.e.ldy, q.e.type, p.yStep, &q.tmaY, &maps[2]));
    RCD_TRY(output(q.e.z, q.e.ldz, q.e.type, p.yStep, &q.tmaZ, &maps[3]));
    RCD_TRY(output(q.e.residual, q.e.ldr, p.form == kScaled ? p.scaling.residualType : q.e.type, p.rStep, &q.tmaR, &maps[4]));
    if (p.symmetric) {                                     // (32 columns of the transpose by 64 of its rows, without the swizzle)
        if (!q.tmaY || yb != 2 || p.M % 64) return fail(ctx, RCD_ERR_INTERNAL, "symmetric products have 16-bit rows of whole pieces");
        RCD_TRY(encode(ctx, &maps[3], map_type(q.e.type), q.e.y, p.N, rows_of(p.yStep), q.e.ldy * yb, 32, 64, CU_TENSOR_MAP_SWIZZLE_NONE));
    }
    q.edgeByHand = !q.raw && p.N * yb % 16 != 0;           // (a piece of the k axis has rows of whole 128 bytes)
    const size_t smem = (size_t)ring.bytes;
    const int slots = plan.pair ? ctx->smCount / 2 : ctx->smCount;
    const int grid = std::min(slots, q.units) * (plan.pair ? 2 : 1);
    const int order = !p.a.across && !p.b.across ? 0 : !p.a.across ? 1 : 2;
    if (p.a.across && !p.b.across) return fail(ctx, RCD_ERR_INTERNAL, "no product takes these orders");
    const int wide = !chunks ? 0 : q.e.type == RCD_ELEM_F32 ? 32 : 64;
    const KernelChoice c = p.form == kPlain ? plain_kernel(i8, order, wide, plan.pair) : p.form == kScaled ? scaled_kernel(order, wide, plan.pair, p.scaling.low && !q.raw) : head_kernel(p.form, p.oneTile, wide, plan.pair);
    const rcd_status rs = run_product(ctx, c, grid, smem, maps, q, st);
    if (rs != RCD_OK || !q.raw) return rs;
    const Scaling scaling = p.form == kScaled ? p.scaling : Scaling{1.0f, 1.0f, nullptr, 0, 0, p.out.type, nullptr};
    const int64_t threads = p.M * ((p.N + 3) / 4);
    return launch_early(ctx, i8 ? join_kernel<true> : join_kernel<false>, dim3((unsigned)((threads + 255) / 256)), 256, st, ws + plan.partAt, plan.splits, (int32_t)p.M, plan.rowsPart,
                        (int32_t)p.N, plan.ldPart, p.out, scaling);
}

}  // namespace rcd

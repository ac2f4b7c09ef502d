// Which tile of a product a unit of work is, and how its operands lie in shared memory (rcd_product.cuh).
#pragma once

#include <algorithm>
#include <cstdint>

#include <cuda_runtime.h>

namespace rcd {

// `tiles` tiles for every piece of the k axis of every matrix of a batch.
struct Walk {
    int32_t tilesM, tilesN, tiles;
    int32_t band;                          // column tiles that are neighbours; the whole width: a row of tiles after the other
    int32_t splits;                        // pieces of the k axis
    int32_t subM, subN;                    // symmetric products: tiles of a square block, down and across; else 0
};
struct Unit {
    int32_t m, n, split, batch;            // tile row and column
    bool mirror;                           // the tile's transpose belongs to the output, too
};

__host__ __device__ inline Unit unit_of(const Walk &w, int32_t u)
{
    Unit t;
    const int32_t piece = u / w.tiles;
    u -= piece * w.tiles;
    t.batch = piece / w.splits;
    t.split = piece - t.batch * w.splits;
    if (w.subM) {
        // Blocks on and below the diagonal, row after row: block (i, j) is number i (i + 1) / 2 + j.
        const int32_t per = w.subM * w.subN, block = u / per, r = u - block * per;
        int32_t i = (int32_t)((sqrtf(8.0f * (float)block + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > block) --i;               // (the root is rounded)
        while ((i + 1) * (i + 2) / 2 <= block) ++i;
        const int32_t j = block - i * (i + 1) / 2;
        t.m = i * w.subM + r / w.subN;
        t.n = j * w.subN + r % w.subN;
        t.mirror = i != j;
        return t;
    }
    // Bands of columns: within one, rows of tiles after one another.
    const int32_t whole = w.tilesM * w.band, at = u / whole, r = u - at * whole;
    const int32_t left = w.tilesN - at * w.band, width = left < w.band ? left : w.band;
    t.m = r / width;
    t.n = at * w.band + (r - t.m * width);
    t.mirror = false;
    return t;
}

constexpr int kOperandRows = 128;          // rows of A per CTA
constexpr int kOperandSlab = 128;          // bytes of k per operand row and stage
constexpr int kOperandStages = 8, kBlockShared = 227 * 1024;

// The ring of operands: stages of aRows + bRows rows, `besides` bytes of other uses behind the last.
struct OperandRing { int32_t stageBytes, stages, bytes; };
inline OperandRing ring_of(int32_t aRows, int32_t bRows, int32_t besides)
{
    OperandRing r;
    r.stageBytes = (aRows + bRows) * kOperandSlab;
    r.stages = std::min(kOperandStages, (kBlockShared - besides) / r.stageBytes);
    // (the instruction reads 128 rows of A wherever a stage begins: those behind few rows have to lie inside, too)
    r.bytes = std::max(r.stages * r.stageBytes + besides, (r.stages - 1) * r.stageBytes + kOperandRows * kOperandSlab);
    return r;
}

}  // namespace rcd

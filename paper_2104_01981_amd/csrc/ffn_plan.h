// Which tiles the products of the feed-forward block take (products.h, ffn.hip), and what of that the kernels have to know.  Host code that
// compiles without HIP, so that tests can ask it.
#pragma once

#include <stddef.h>

#include "element.h"

namespace ecrm {

constexpr uint32_t kRowBytes = 128;              // of K, in a tile
constexpr uint32_t kAtOnce = 4;                  // steps of 64 bytes of K that a wave of few rows' products has in flight

// ---- which tiles -----------------------------------------------------------------------------------------------------------------
// What a product takes is estimated in us from what was measured (M, N of 512 to 4096, all CUs in step): a tile's steps of 128 bytes of
// K, alone on its CU and for each of several (times `transposed` for the gradients in 16 bits); the launch, a tile's begin and end (`back`: kBack's,
// which is bound by what it reads and writes).  16 bits: 64 x 64 0.50 and 0.17 a step, 128 x 128 0.65
// and 0.47, 256 x 256 1.58.  32 bits are bound by their matrix instructions, 137 TFLOP/s with any of these and all CUs full, so that small
// tiles, more of them to a CU, gain: 32 x 32 0.24 and 0.12, 64 x 64 0.62 and 0.46, 128 x 128 1.96 and 1.79 (777 rows, D = 260, F =
// 684: 26 us with 64 x 64 at least, 19 so).
enum { kTile256 = 0, kTile128 = 1, kTile64 = 2, kTile32 = 3, kTilings = 4 };
struct TilingCost { uint32_t side, resident; double step[2], shared[2], transposed, launch, tile, back; };      // [0] 16 bits, [1] 32; 0: not for these
constexpr TilingCost kCosts[kTilings] = {{256, 1, {1.58, 0}, {1.58, 0}, 1.0, 3.0, 8.0, 20.0}, {128, 2, {0.65, 1.96}, {0.47, 1.79}, 1.06, 5.0, 1.4, 6.8},
                                         {64, 5, {0.50, 0.62}, {0.172, 0.46}, 1.25, 2.5, 0.42, 1.6}, {32, 8, {0, 0.24}, {0, 0.12}, 1.0, 2.5, 0.3, 0.6}};
// Columns of a tile; of each projection for kGate.
constexpr uint32_t columns_of(uint32_t side, bool dual) { return dual && side > 32 ? side / 2u : side; }
constexpr uint32_t kSkinnyParts = 16;
constexpr size_t kPartMost = 32u << 20;          // bytes of the parts of split products, at most
constexpr uint32_t kCounters = kPartMost / (2u * 32u * 32u * 4u);       // tiles of two parts or more

struct Split { uint32_t splits, each; };
// Products of one launch (the last of them with the splits of their own, where there are two sizes).
struct Plan { uint32_t tiling; Split split[2]; uint32_t counters; double cost; };
// Rows up to `rows` of the results with one tiling, the others (if there are any) with another.
struct RowPlan { uint32_t rows; Plan main, rest; };

struct ProductSize { uint32_t M, N, K, halves, count; bool dual, first, gradients; };       // `count` of them

// Up to 32 rows, of 32 bits up to 16, are skinny_kernel's.  us forward so / by tiles, 16 and 32 rows: bf16 D = 128, F = 512 6.8 / 8.7, 8.2 /
// 8.7; 1024, 1024 9.2 / 14.5, 11.5 / 14.6; 1024, 4096 15.1 / 19.8, 20.1 / 19.8.  fp32 8.0 / 12.6, 10.0 / 12.7; 15.2 / 21.4, 23.5 / 21.3;
// 29.2 / 31.5, 44.3 / 31.4.
inline uint32_t skinny_waves(uint32_t K, uint32_t type)        // that have kAtOnce steps each
{
    const uint32_t steps = (K * type_bytes(type) + 63u) / 64u;
    return (steps + kAtOnce - 1u) / kAtOnce;
}
inline uint32_t skinny_parts(uint32_t N, uint32_t K, uint32_t type, uint32_t cus)
{
    const uint32_t blocks = (N + 15u) / 16u, fit = cus / blocks, fill = skinny_waves(K, type) / 8u;
    const uint32_t parts = fit < fill ? fit : fill;      // no more workgroups than CUs, eight waves at least to each
    return parts < 1u ? 1u : parts > kSkinnyParts ? kSkinnyParts : parts;
}
inline bool is_skinny(uint32_t rows, uint32_t type) { return rows <= (type == ECRM_F32 ? 16u : 32u); }

Plan plan_launch(const ProductSize &a, const ProductSize &b, uint32_t type, uint32_t cus, size_t room);
RowPlan plan_rows(const ProductSize &other, const ProductSize &z, uint32_t type, uint32_t cus, size_t room);

// What of a block is planned at a time: the launches of a forward pass (gate and out); of a backward pass the gradient of h, and those of the
// weights alone, of x alone, or of both side by side.
enum { kPlanForward, kPlanBack, kPlanWeights, kPlanInput, kPlanBoth, kPlans };
struct BlockPlans { RowPlan gate, out, back, weights, input, both; };
void plan_block(BlockPlans &plans, int what, uint32_t rows, uint32_t dim, uint32_t hidden, uint32_t type, uint32_t cus, size_t room);
// Bytes of parts, kPartMost at most, that no plan of a block of up to max_rows rows is the worse for, whatever the number of CUs.
size_t parts_room(uint32_t dim, uint32_t hidden, uint64_t max_rows, uint32_t type, bool training);

// false: more workgroups than a launch can have, of any tiling
inline bool is_planned(const RowPlan &p) { return p.main.cost > 0; }
inline uint32_t counters_of(const RowPlan &p) { return p.main.counters > p.rest.counters ? p.main.counters : p.rest.counters; }

}  // namespace ecrm

// Plans of the feed-forward block's products: see ffn_plan.h.  Host code only, without HIP.
#include "ffn_plan.h"

#include <initializer_list>

namespace ecrm {

constexpr uint32_t kSplitCounts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}, kMostParts = 64;
// Parts joined by the workgroup that is there last: us; bytes of parts a us, of one tile's and, in 16 bits, of all.  Without the last, bf16,
// backward of 8192 rows, D = 512, F = 2048 174 us instead of 144, of 4096, 256 x 1024 42.6 instead of 36.6, forward of 2000 of these 21.2
// instead of 18.4; it costs forward of 4096, 1024 x 4096 3 % and backward of 16384, 260 x 684 9 %.  In 32 bits, whose tiles take longer,
// it would cost forward of 600 rows, 260 x 684 18.6 -> 20.6 and gain nothing.
constexpr double kJoinWait = 2.0, kJoinOne = 2.5e4, kJoinAll = 1e7;
constexpr uint64_t kMostWorkgroups = 0xFFFFFFFFu / 512u;        // a launch has fewer than 2^32 threads

constexpr double kSkinnyLaunch = 3.5, kSkinnyRate = 2.5e6;               // us; bytes of weights a us

static uint64_t tiles_of(const ProductSize &z, uint32_t M, uint32_t side)
{
    const uint32_t columns = columns_of(side, z.dual);
    return (uint64_t)((M + side - 1) / side) * ((z.N + columns - 1) / columns) * z.count;
}

// What a launch of A tiles that take ta and then B that take tb, so many at a time, takes.
static double makespan(uint64_t A, double ta, uint64_t B, double tb, uint64_t slots)
{
    // the places that have one of the first kind more than the others, and those others
    uint64_t n[2] = {A % slots, slots - A % slots};
    double at[2] = {(double)(A / slots + 1) * ta, (double)(A / slots) * ta}, end = n[0] ? at[0] : at[1];
    while (B) {
        const int g = n[0] && at[0] <= at[1] ? 0 : 1;
        at[g] += tb;
        if (at[g] > end) end = at[g];
        B -= B < n[g] ? B : n[g];
    }
    return end;
}

// The sizes' products side by side (b.count = 0: a alone).
Plan plan_launch(const ProductSize &a, const ProductSize &b, uint32_t type, uint32_t cus, size_t room)
{
    const uint32_t wide = type == ECRM_F32 ? 1u : 0u, elements = kRowBytes / type_bytes(type);
    const ProductSize *sizes[2] = {&a, &b};
    Plan best{};
    for (uint32_t t = 0; t < kTilings; ++t) {
        const TilingCost &c = kCosts[t];
        if (c.step[wide] == 0.0) continue;
        uint64_t tiles[2];
        uint32_t k_tiles[2];
        for (int i = 0; i < 2; ++i) {
            tiles[i] = sizes[i]->count ? tiles_of(*sizes[i], sizes[i]->M, c.side) : 0;
            k_tiles[i] = (sizes[i]->K + elements - 1) / elements * sizes[i]->halves;
        }
        auto split = [&](int i, uint32_t splits) {
            const uint32_t each = (k_tiles[i] + splits - 1) / splits;
            return Split{(k_tiles[i] + each - 1) / each, each};
        };
        const double part = (double)c.side * c.side * 4.0;
        for (uint32_t sa : kSplitCounts) {
            if (sa > k_tiles[0] || (a.first && sa > 1)) break;           // a call's first product has no counters that are cleared before it
            const Split x = split(0, sa);
            const double a_bytes = x.splits > 1 ? part * tiles[0] * x.splits : 0.0;
            if (a_bytes > (double)room) break;
            for (uint32_t sb : kSplitCounts) {
                if (b.count ? sb > k_tiles[1] : sb > 1) break;
                const Split y = b.count ? split(1, sb) : Split{1, 0};
                const double bytes = a_bytes + (y.splits > 1 ? part * tiles[1] * y.splits : 0.0);
                if (bytes > (double)room) break;
                const uint64_t units = tiles[0] * x.splits + tiles[1] * y.splits, there = (units + cus - 1) / cus;
                if (units > kMostWorkgroups) continue;
                const double together = there < c.resident ? (double)there : (double)c.resident;
                // 32 x 32 of each projection are twice the work, larger tiles have both in their width
                const double twice = a.dual && c.side == 32 ? 2.0 : 1.0;
                const double alone = c.step[wide] * twice, shared = c.shared[wide] * twice * together * (a.gradients && !wide ? c.transposed : 1.0);
                const double step = shared > alone ? shared : alone;
                auto unit = [&](int i, const Split &s) {
                    return (a.first && !a.dual ? c.back : c.tile) * together + s.each * step + (s.splits > 1 ? kJoinWait + s.splits * part / kJoinOne : 0.0);
                };
                const uint64_t slots = (uint64_t)(cus * together);
                const double ua = unit(0, x), ub = b.count ? unit(1, y) : 1.0;
                double cost = c.launch + (wide ? 0.0 : bytes / kJoinAll) + (ua >= ub ? makespan(tiles[0] * x.splits, ua, tiles[1] * y.splits, ub, slots)
                                                                                       : makespan(tiles[1] * y.splits, ub, tiles[0] * x.splits, ua, slots));
                const uint64_t counters = (x.splits > 1 ? tiles[0] : 0) + (y.splits > 1 ? tiles[1] : 0);
                if (!best.split[0].splits || cost < best.cost) best = Plan{t, {x, y}, (uint32_t)counters, cost};
            }
        }
    }
    return best;
}

// z's products with its rows cut where that is faster, those up to the cut beside the other size's (other.count = 0: alone).
RowPlan plan_rows(const ProductSize &other, const ProductSize &z, uint32_t type, uint32_t cus, size_t room)
{
    const ProductSize none{};
    auto plan = [&](uint32_t rows, bool beside) {
        ProductSize part = z;
        part.M = rows;
        if (!z.gradients && (z.dual || !z.first) && is_skinny(rows, type)) {
            Plan skinny{};
            skinny.cost = kSkinnyLaunch + (double)z.N * z.K * (z.dual ? 2 : 1) * type_bytes(type) / kSkinnyRate;
            return skinny;
        }
        return beside && other.count ? plan_launch(other, part, type, cus, room) : plan_launch(part, none, type, cus, room);
    };
    RowPlan best{z.M, plan(z.M, true), Plan{}};
    for (uint32_t side : {256u, 128u, 64u}) {
        // as many rows of tiles as fill the CUs to the last, or as are whole
        const uint64_t across = tiles_of(z, side, side), all = z.M / side, rounds = all * across / cus;
        for (uint64_t down : {rounds * cus / across, all}) {
            const uint32_t rows = (uint32_t)(down * side);
            if (!rows || rows >= z.M) continue;
            const Plan main = plan(rows, true), rest = plan(z.M - rows, false);
            if (main.cost + rest.cost < best.main.cost + best.rest.cost) best = RowPlan{rows, main, rest};
        }
    }
    return best;
}

void plan_block(BlockPlans &plans, int what, uint32_t rows, uint32_t dim, uint32_t hidden, uint32_t type, uint32_t cus, size_t room)
{
    const ProductSize none{}, weights{hidden, dim, rows, 1, 3, false, false, true}, input{rows, dim, hidden, 2, 1, false, false, true};
    if (what == kPlanForward) {
        plans.gate = plan_rows(none, ProductSize{rows, hidden, dim, 1, 1, true, true, false}, type, cus, room);
        plans.out = plan_rows(none, ProductSize{rows, dim, hidden, 1, 1, false, false, false}, type, cus, room);
    } else if (what == kPlanBack) {
        plans.back = plan_rows(none, ProductSize{rows, hidden, dim, 1, 1, false, true, false}, type, cus, room);
    } else if (what == kPlanWeights) {
        plans.weights = RowPlan{hidden, plan_launch(weights, none, type, cus, room), Plan{}};
    } else if (what == kPlanInput) {
        plans.input = plan_rows(none, input, type, cus, room);
    } else {
        plans.both = plan_rows(weights, input, type, cus, room);
    }
}

size_t parts_room(uint32_t dim, uint32_t hidden, uint64_t max_rows, uint32_t type, bool training)
{
    const uint32_t rows = (uint32_t)max_rows, wide = type == ECRM_F32 ? 1u : 0u, elements = kRowBytes / type_bytes(type);
    uint64_t most = 0;
    for (uint32_t t = 0; t < kTilings; ++t) {
        const TilingCost &c = kCosts[t];
        if (c.step[wide] == 0.0) continue;
        // all tiles in as many parts as there may be
        auto parts = [&](const ProductSize &z) {
            const uint64_t k_tiles = (uint64_t)((z.K + elements - 1) / elements) * z.halves, cut = k_tiles < kMostParts ? k_tiles : kMostParts;
            return cut > 1 ? tiles_of(z, z.M, c.side) * cut * c.side * c.side * 4u : 0u;
        };
        const uint64_t out = is_skinny(rows, type) ? 0 : parts(ProductSize{rows, dim, hidden, 1, 1, false, false, false});
        const uint64_t gradients = training ? parts(ProductSize{hidden, dim, rows, 1, 3, false, false, true}) +
                                                  parts(ProductSize{rows, dim, hidden, 2, 1, false, false, true}) : 0;
        most = out > most ? out : most;
        most = gradients > most ? gradients : most;
    }
    // few rows: 1 KB for each of up to two blocks of 16 rows and of 16 columns
    const uint32_t waves = skinny_waves(hidden, type) / 8u;
    const uint64_t few = waves > 1 ? (uint64_t)((dim + 15u) / 16u) * (waves < kSkinnyParts ? waves : kSkinnyParts) * 2048u : 0;
    most = few > most ? few : most;
    return most < kPartMost ? (size_t)most : kPartMost;
}

}  // namespace ecrm

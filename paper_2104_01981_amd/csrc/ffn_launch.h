// Launches of the feed-forward block's products as planned, for a type (ffn_block.h).
#pragma once

#include "ffn_block.h"

namespace ecrm {

template <typename T>
constexpr uint32_t type_of() { return sizeof(T) == 4 ? ECRM_F32 : ECRM_BF16; }       // of either type of 16 bits plans are the same

// Gives the products of a launch their tiles, parts and workgroups, in order.
static void lay_out(ProductArgs &a, uint32_t rows, uint32_t columns)
{
    a.workgroups = 0;
    uint32_t part = 0, counter = 0;
    for (uint32_t i = 0; i < a.products; ++i) {
        Product &p = a.p[i];
        p.tiles_m = (p.M + rows - 1) / rows;
        p.tiles_n = (p.N + columns - 1) / columns;
        const uint32_t tiles = p.tiles_m * p.tiles_n;
        p.first = a.workgroups;
        a.workgroups += tiles * p.splits;
        if (p.splits == 1) continue;
        p.part = part;
        p.counter = counter;
        part += tiles * p.splits;
        counter += tiles;
    }
}

template <typename T, int KIND, int BM, int BN, int WM, int WN>
static void launch_tiling(ProductArgs &a, hipStream_t st)
{
    typedef Tiling<T, KIND, BM, BN, WM, WN> L;
    lay_out(a, BM, L::kColumns);
    hipLaunchKernelGGL((product_kernel<T, KIND, BM, BN, WM, WN>), dim3(a.workgroups), dim3(L::kThreads), 0, st, a);
}

template <typename T, int KIND>
static void launch_planned(ProductArgs &a, const Plan &plan, hipStream_t st)
{
    a.products = 1;
    a.p[0].splits = plan.split[0].splits;
    a.p[0].each = plan.split[0].each;
    // both projections of kGate: 64 columns of each to a wave (32 of 64 x 64), whole lines of the results
    if constexpr (sizeof(T) == 2) {
        if (plan.tiling == kTile256) {
            if constexpr (KIND == kGate) launch_tiling<T, KIND, 256, 256, 4, 2>(a, st);
            else launch_tiling<T, KIND, 256, 256, 2, 4>(a, st);
            return;
        }
    }
    if constexpr (sizeof(T) == 4) {
        if (plan.tiling == kTile32) {
            if constexpr (KIND == kGate) launch_tiling<T, KIND, 32, 64, 2, 2>(a, st);
            else launch_tiling<T, KIND, 32, 32, 2, 2>(a, st);
            return;
        }
    }
    if (plan.tiling == kTile128) {
        if constexpr (KIND == kGate) launch_tiling<T, KIND, 128, 128, 4, 1>(a, st);
        else launch_tiling<T, KIND, 128, 128, 2, 2>(a, st);
    } else {
        if constexpr (KIND == kGate) launch_tiling<T, KIND, 64, 64, 4, 1>(a, st);
        else launch_tiling<T, KIND, 64, 64, 2, 2>(a, st);
    }
}

template <typename T, int BM, int BN, int WM, int WN>
static void launch_gradients(ProductArgs &a, hipStream_t st)
{
    lay_out(a, BM, BN);
    hipLaunchKernelGGL((gradients_kernel<T, BM, BN, WM, WN>), dim3(a.workgroups), dim3(WM * WN * kWave), 0, st, a);
}

// The weights' products, those of x, or both.
template <typename T>
static void launch_gradients(ProductArgs &a, const Product *weights, const Product *input, const Plan &plan, hipStream_t st)
{
    a.products = 0;
    auto take = [&](const Product *p, uint32_t count, const Split &s) {
        for (uint32_t i = 0; i < count; ++i) {
            Product &to = a.p[a.products++];
            to = p[i];
            to.splits = s.splits;
            to.each = s.each;
        }
    };
    // longest first
    if (weights && input && plan.split[0].each < plan.split[1].each) {
        take(input, 1, plan.split[1]);
        take(weights, 3, plan.split[0]);
    } else {
        if (weights) take(weights, 3, plan.split[0]);
        if (input) take(input, 1, plan.split[weights ? 1 : 0]);
    }
    if constexpr (sizeof(T) == 2)
        if (plan.tiling == kTile256) return launch_gradients<T, 256, 256, 2, 4>(a, st);
    if constexpr (sizeof(T) == 4)
        if (plan.tiling == kTile32) return launch_gradients<T, 32, 32, 2, 2>(a, st);
    if (plan.tiling == kTile128) launch_gradients<T, 128, 128, 2, 2>(a, st);
    else launch_gradients<T, 64, 64, 2, 2>(a, st);
}

// The product's rows from `first` on.
template <typename T, int KIND>
static void skip_rows(ProductArgs &a, uint32_t first)
{
    Product &p = a.p[0];
    auto on = [&](const void *q, uint64_t stride) { return q ? (void *)((T *)q + first * stride) : nullptr; };
    for (int i = 0; i < 2; ++i) p.a.p[i] = on(p.a.p[i], p.a.stride[i]);
    p.out = on(p.out, p.out_stride);
    if (KIND == kGate) p.out2 = on(p.out2, 2ull * p.N);
    if (KIND == kBack) {
        p.in = on(p.in, 2ull * p.N);
        p.out2 = on(p.out2, p.out_stride);
        p.out3 = on(p.out3, p.out_stride);
    } else {
        p.in = on(p.in, p.in_stride);
    }
    a.first_row = first;
    p.M -= first;
}

template <typename T, int KIND, int XB>
static void launch_skinny(ProductArgs &a, uint32_t cus, hipStream_t st)
{
    constexpr uint32_t type = type_of<T>();
    const Product &p = a.p[0];
    const uint32_t parts = KIND == kOut ? skinny_parts(p.N, p.K, type, cus) : 1u, share = (skinny_waves(p.K, type) + parts - 1u) / parts;
    const uint32_t waves = share < Skinny<XB>::kWaves ? share : Skinny<XB>::kWaves;
    hipLaunchKernelGGL((skinny_kernel<T, KIND, XB>), dim3((p.N + 15u) / 16u, parts), dim3(waves * kWave), 0, st, a);
}

template <typename T, int KIND>
static void launch_rows(ProductArgs &a, const Plan &plan, uint32_t cus, hipStream_t st)
{
    if constexpr (KIND == kGate || KIND == kOut) {
        if (is_skinny(a.p[0].M, type_of<T>())) {
            if (a.p[0].M <= 16) return launch_skinny<T, KIND, 1>(a, cus, st);
            if constexpr (sizeof(T) == 2) return launch_skinny<T, KIND, 2>(a, cus, st);
        }
    }
    launch_planned<T, KIND>(a, plan, st);
}

template <typename T, int KIND>
static void launch_product(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st)
{
    const uint32_t M = a.p[0].M;
    a.first_row = 0;
    a.p[0].M = plan.rows;
    launch_rows<T, KIND>(a, plan.main, cus, st);
    if (plan.rows == M) return;
    a.p[0].M = M;
    skip_rows<T, KIND>(a, plan.rows);
    launch_rows<T, KIND>(a, plan.rest, cus, st);
}

template <typename T>
void BlockLaunch<T>::gate(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st) { launch_product<T, kGate>(a, plan, cus, st); }
template <typename T>
void BlockLaunch<T>::out(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st) { launch_product<T, kOut>(a, plan, cus, st); }
template <typename T>
void BlockLaunch<T>::back(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st) { launch_product<T, kBack>(a, plan, cus, st); }

template <typename T>
void BlockLaunch<T>::gradients(ProductArgs &a, const Product *weights, const Product *input, const RowPlan &plan, hipStream_t st)
{
    if (!input) return launch_gradients<T>(a, weights, nullptr, plan.main, st);
    Product in = *input;
    in.M = plan.rows;
    launch_gradients<T>(a, weights, &in, plan.main, st);
    if (plan.rows == input->M) return;
    a.p[0] = *input;
    skip_rows<T, kInput>(a, plan.rows);
    in = a.p[0];
    launch_gradients<T>(a, nullptr, &in, plan.rest, st);
}

}  // namespace ecrm

// The feed-forward block's launches as planned, of one type: a source of its own for each (ffn_bf16.hip and so on), since compiling them takes
// most of the build.
#pragma once

#include "ffn_plan.h"
#include "products.h"

namespace ecrm {

template <typename T>
struct BlockLaunch {
    static void gate(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st);
    static void out(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st);
    static void back(ProductArgs &a, const RowPlan &plan, uint32_t cus, hipStream_t st);
    // the products of the weights, those of x, or both (one or the other may be null), x's rows as planned
    static void gradients(ProductArgs &a, const Product *weights, const Product *input, const RowPlan &plan, hipStream_t st);
};

}  // namespace ecrm

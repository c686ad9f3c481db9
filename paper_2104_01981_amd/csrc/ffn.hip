// The gated feed-forward block and its gradients: h = act(x Wg^T) * (x Wu^T) in one launch, out = residual + drop(h Wd^T) in a second;
// backward, from the gradient of out: what the mask keeps of it (a launch with dropout), dg, du and h in the epilogue of the gradient of h
// (one), the gradients of the three weights and of x side by side (one).  g and u are saved, not computed again: two products in six.
//
// What bounds it.  Large batches: the matrix cores, 16 411 rows with D = 1024 and F = 4096 in bf16 forward 405 to 440 us (1020 to 940 TFLOP/s,
// with 0.27 GB of g and u written on the way), backward 900 to 955 (920 to 860); the same products alone take the library 515 and 1215 us.  kBack is bound by
// memory instead: two elements in and three out for each of h, 245 us, 105 of them multiplications.  D = 128, F = 512, 8192
// rows: memory, 16 us forward, of which g, u and h take 6; 33 backward.  A few rows: the weights, 25 MB for five rows in 11 us.
#include "ffn_block.h"

#include <new>
#include <string.h>

namespace ecrm {

__global__ __launch_bounds__(256) void clear_kernel(uint32_t *to, uint64_t words)
{
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < words; i += (uint64_t)gridDim.x * 256u) to[i] = 0u;
}

}  // namespace ecrm

using namespace ecrm;

// ---- C ABI -----------------------------------------------------------------------------------------------------------------------
struct ecrm_ffn {
    ecrm_ffn_config cfg;
    uint64_t pitch;                       // elements of a row of h, dg, du
    uint64_t e_pitch;                     // of a row of e
    size_t off_h, off_dg, off_du, off_e, off_arrived, off_part, part_bytes, bytes;
    const void *gate_weights, *up, *down;
    uint64_t gate_stride, up_stride, down_stride;
    char *work;
    int cus;
    // plans, kept while the number of rows stays, since making them takes some us
    uint64_t rows_of[kPlans];
    BlockPlans plans;
};

namespace {

constexpr uint64_t kStrideMost = 1u << 20;

struct Rows { const void *p; uint64_t rows, cols, stride; };     // elements

// Rows of the workspace: no power of two apart, or a tile's rows lie behind one another in the same channel of a cache (16384 x 4096 x
// 4096 in bf16 with both operands' rows 8 KB apart 437-466 us, with 8.375 KB 416; 8.125 KB lies between).
uint64_t pitch_of(uint64_t elements, uint64_t size)
{
    const uint64_t bytes = elements * size;
    return ((bytes <= 384 ? 0 : (bytes - 384 + 511) / 512 * 512) + 384) / size;
}

bool rows_fit(const ecrm_ffn *f, const Rows &r)
{
    const uint32_t size = type_bytes(f->cfg.type);
    return r.p && (uintptr_t)r.p % (4 * size) == 0 && r.stride >= r.cols && r.stride % 4 == 0 && r.stride <= kStrideMost;
}

bool apart(uint32_t a_size, const Rows &a, uint32_t b_size, const Rows &b)
{
    return strided_apart(a.p, a.p ? a.rows : 0, a.cols * a_size, a.stride * a_size, b.p, b.p ? b.rows : 0, b.cols * b_size, b.stride * b_size);
}

// Is what is read clear of the workspace, which is written?
bool clear_of_work(const ecrm_ffn *f, const Rows &r) { return apart(type_bytes(f->cfg.type), r, 1, Rows{f->work, 1, f->bytes, f->bytes}); }

bool mask_fits(const ecrm_ffn *f, const ecrm_mask *mask, MaskArgs &to)
{
    double factor;
    return make_mask(mask, to, factor) && apart(1, Rows{mask->state, 1, 16, 16}, 1, Rows{f->work, 1, f->bytes, f->bytes});
}

// Is what is written clear of the weights, the workspace and the mask's state?
bool clear_of_own(const ecrm_ffn *f, const ecrm_mask *mask, uint32_t size, const Rows &w)
{
    const uint32_t s = type_bytes(f->cfg.type);
    const uint64_t D = f->cfg.dim, F = f->cfg.hidden;
    return apart(size, w, s, Rows{f->gate_weights, F, D, f->gate_stride}) && apart(size, w, s, Rows{f->up, F, D, f->up_stride}) &&
           apart(size, w, s, Rows{f->down, D, F, f->down_stride}) && apart(size, w, 1, Rows{f->work, 1, f->bytes, f->bytes}) &&
           (!mask || apart(size, w, 1, Rows{mask->state, 1, 16, 16}));
}

int launched() { return hipGetLastError() == hipSuccess ? ECRM_OK : ECRM_EHIP; }

Product product(const void *a, uint64_t a_stride, const void *b, uint64_t b_stride, uint32_t M, uint32_t N, uint32_t K)
{
    Product p;
    memset(&p, 0, sizeof(p));
    p.a.p[0] = p.a.p[1] = a;
    p.a.stride[0] = p.a.stride[1] = a_stride;
    p.b.p[0] = p.b.p[1] = b;
    p.b.stride[0] = p.b.stride[1] = b_stride;
    p.M = M; p.N = N; p.K = K;
    p.scale = 1.0f;
    return p;
}

void make_plan(ecrm_ffn *f, int what, uint32_t n)
{
    if (f->rows_of[what] == n) return;
    plan_block(f->plans, what, n, f->cfg.dim, f->cfg.hidden, f->cfg.type, (uint32_t)f->cus, f->part_bytes);
    f->rows_of[what] = n;
}

}  // namespace

extern "C" {

int ecrm_ffn_create(const ecrm_ffn_config *cfg, ecrm_ffn **out)
{
    if (!out) return ECRM_EINVAL;
    *out = nullptr;
    if (!cfg || cfg->dim < 4 || cfg->dim % 4 || cfg->dim > 65536 || cfg->hidden < 4 || cfg->hidden % 4 || cfg->hidden > 65536) return ECRM_EINVAL;
    if (cfg->type > ECRM_F16 || cfg->activation > ECRM_RELU || cfg->training > 1) return ECRM_EINVAL;
    if (!cfg->max_rows || cfg->max_rows > (1ull << 26)) return ECRM_EINVAL;
    ecrm_ffn *f = new (std::nothrow) ecrm_ffn;
    if (!f) return ECRM_EINVAL;
    memset(f, 0, sizeof(*f));
    f->cfg = *cfg;
    const uint64_t size = type_bytes(cfg->type), D = cfg->dim, F = cfg->hidden;
    f->pitch = pitch_of(F, size);
    f->e_pitch = pitch_of(D, size);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    f->off_h = take(cfg->max_rows * f->pitch * size);
    if (cfg->training) {
        f->off_dg = take(cfg->max_rows * f->pitch * size);
        f->off_du = take(cfg->max_rows * f->pitch * size);
        f->off_e = take(cfg->max_rows * f->e_pitch * size);
    }
    f->off_arrived = take(((cfg->dim + 15u) / 16u * 2u > kCounters ? (cfg->dim + 15u) / 16u * 2u : kCounters) * 4u);
    f->part_bytes = parts_room(cfg->dim, cfg->hidden, cfg->max_rows, cfg->type, cfg->training != 0);
    f->off_part = take(f->part_bytes);
    f->bytes = off;
    *out = f;
    return ECRM_OK;
}

void ecrm_ffn_destroy(ecrm_ffn *f) { delete f; }

size_t ecrm_ffn_bytes(const ecrm_ffn *f) { return f ? f->bytes : 0; }

int ecrm_ffn_bind(ecrm_ffn *f, const void *gate, uint64_t gate_stride, const void *up, uint64_t up_stride, const void *down,
                  uint64_t down_stride, void *work, size_t work_bytes)
{
    if (!f) return ECRM_EINVAL;
    const uint64_t D = f->cfg.dim, F = f->cfg.hidden;
    const Rows g{gate, F, D, gate_stride}, u{up, F, D, up_stride}, d{down, D, F, down_stride};
    if (!rows_fit(f, g) || !rows_fit(f, u) || !rows_fit(f, d)) return ECRM_EINVAL;
    if (!work || (uintptr_t)work % 256 || work_bytes < f->bytes) return ECRM_ESCRATCH;
    const Rows w{work, 1, f->bytes, f->bytes};
    const uint32_t size = type_bytes(f->cfg.type);
    if (!apart(1, w, size, g) || !apart(1, w, size, u) || !apart(1, w, size, d)) return ECRM_EINVAL;
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
        return ECRM_EHIP;
    f->gate_weights = gate; f->up = up; f->down = down;
    f->gate_stride = gate_stride; f->up_stride = up_stride; f->down_stride = down_stride;
    f->work = (char *)work;
    f->cus = cus;
    memset(f->rows_of, 0, sizeof(f->rows_of));
    return ECRM_OK;
}

int ecrm_ffn_forward(ecrm_ffn *f, const void *x, uint64_t x_stride, uint64_t n, const void *residual, uint64_t residual_stride,
                     const ecrm_mask *mask, void *out, uint64_t out_stride, void *saved, void *stream)
{
    if (!f) return ECRM_EINVAL;
    if (!f->work) return ECRM_ENOTBOUND;
    if (n > f->cfg.max_rows) return ECRM_EBATCH;
    ProductArgs a;
    memset(&a, 0, sizeof(a));
    if (mask && !mask_fits(f, mask, a.mask)) return ECRM_EINVAL;
    if (!n) return ECRM_OK;
    const uint32_t D = f->cfg.dim, F = f->cfg.hidden, N = (uint32_t)n, type = f->cfg.type, size = type_bytes(type);
    if (n == 1) x_stride = residual_stride = out_stride = D;             // of one row it says nothing
    const Rows rx{x, n, D, x_stride}, rr{residual, n, D, residual_stride}, ro{out, n, D, out_stride}, rs{saved, n, 2ull * F, 2ull * F};
    if (!rows_fit(f, rx) || !rows_fit(f, ro) || (residual && !rows_fit(f, rr))) return ECRM_EINVAL;
    if (saved && (uintptr_t)saved % (4 * size)) return ECRM_EINVAL;
    auto in_place = [&](const Rows &r) { return r.p == out && r.stride == out_stride; };
    if ((!in_place(rx) && !apart(size, rx, size, ro)) || (residual && !in_place(rr) && !apart(size, rr, size, ro))) return ECRM_EINVAL;
    if (!clear_of_own(f, mask, size, ro) || !clear_of_work(f, rx) || !clear_of_work(f, rr)) return ECRM_EINVAL;
    if (saved && (!apart(size, rs, size, rx) || !apart(size, rs, size, rr) || !apart(size, rs, size, ro) || !clear_of_own(f, mask, size, rs)))
        return ECRM_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    void *h = f->work + f->off_h;
    a.part = (float *)(f->work + f->off_part);
    make_plan(f, kPlanForward, N);
    if (!is_planned(f->plans.gate) || !is_planned(f->plans.out)) return ECRM_EINVAL;
    a.arrived = (uint32_t *)(f->work + f->off_arrived);
    a.clear = counters_of(f->plans.out);
    if (is_skinny(f->plans.out.rows < N ? N - f->plans.out.rows : N, type) && skinny_parts(D, F, type, (uint32_t)f->cus) > 1 &&
        a.clear < (D + 15u) / 16u * 2u)
        a.clear = (D + 15u) / 16u * 2u;
    a.activation = f->cfg.activation;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        a.p[0] = product(x, x_stride, f->gate_weights, f->gate_stride, N, F, D);
        a.p[0].b.p[1] = f->up;
        a.p[0].b.stride[1] = f->up_stride;
        a.p[0].out = h;
        a.p[0].out_stride = f->pitch;
        a.p[0].out2 = saved;
        BlockLaunch<T>::gate(a, f->plans.gate, (uint32_t)f->cus, st);
        a.p[0] = product(h, f->pitch, f->down, f->down_stride, N, D, F);
        a.p[0].out = out;
        a.p[0].out_stride = out_stride;
        a.p[0].in = residual;
        a.p[0].in_stride = residual_stride;
        a.masked = mask ? 1u : 0u;
        BlockLaunch<T>::out(a, f->plans.out, (uint32_t)f->cus, st);
    });
    return launched();
}

int ecrm_ffn_backward(ecrm_ffn *f, const void *x, uint64_t x_stride, const void *saved, const void *d_out, uint64_t d_out_stride,
                      uint64_t n, const ecrm_mask *mask, const void *add, uint64_t add_stride, void *d_x, uint64_t d_x_stride,
                      void *d_gate, void *d_up, void *d_down, uint32_t weight_type, int accumulate, void *stream)
{
    if (!f) return ECRM_EINVAL;
    if (!f->work) return ECRM_ENOTBOUND;
    if (!f->cfg.training) return ECRM_ESCRATCH;
    if (n > f->cfg.max_rows) return ECRM_EBATCH;
    ProductArgs a;
    memset(&a, 0, sizeof(a));
    if (mask && !mask_fits(f, mask, a.mask)) return ECRM_EINVAL;
    const uint32_t D = f->cfg.dim, F = f->cfg.hidden, N = (uint32_t)n, type = f->cfg.type, size = type_bytes(type);
    const bool weights = d_gate || d_up || d_down;
    const uint32_t weight_size = type_bytes(weight_type);
    const Rows rg{d_gate, F, D, D}, ru{d_up, F, D, D}, rd{d_down, D, F, F};
    if (weights) {
        if (!d_gate || !d_up || !d_down || (weight_type != type && weight_type != ECRM_F32)) return ECRM_EINVAL;
        for (const Rows *r : {&rg, &ru, &rd})
            if ((uintptr_t)r->p % (4 * weight_size) || !clear_of_own(f, mask, weight_size, *r)) return ECRM_EINVAL;
        if (!apart(weight_size, rg, weight_size, ru) || !apart(weight_size, rg, weight_size, rd) || !apart(weight_size, ru, weight_size, rd)) return ECRM_EINVAL;
    }
    hipStream_t st = (hipStream_t)stream;
    if (!n) {
        if (weights && !accumulate)
            for (void *p : {d_gate, d_up, d_down})
                hipLaunchKernelGGL(clear_kernel, dim3((uint32_t)f->cus), dim3(256), 0, st, (uint32_t *)p, (uint64_t)D * F * weight_size / 4u);
        return launched();
    }
    if (n == 1) x_stride = d_out_stride = add_stride = d_x_stride = D;   // of one row it says nothing
    const Rows rx{x, n, D, x_stride}, rs{saved, n, 2ull * F, 2ull * F}, ro{d_out, n, D, d_out_stride}, ra{d_x ? add : nullptr, n, D, add_stride},
        rdx{d_x, n, D, d_x_stride};
    if (!rows_fit(f, rx) || !rows_fit(f, ro) || (d_x && !rows_fit(f, rdx)) || (ra.p && !rows_fit(f, ra))) return ECRM_EINVAL;
    if (!saved || (uintptr_t)saved % (4 * size)) return ECRM_EINVAL;
    for (const Rows *r : {&rx, &rs, &ro, &ra})
        if (!clear_of_work(f, *r)) return ECRM_EINVAL;
    if (weights)
        for (const Rows *w : {&rg, &ru, &rd})
            for (const Rows *r : {&rx, &rs, &ro, &ra, &rdx})
                if (!apart(weight_size, *w, size, *r)) return ECRM_EINVAL;
    if (d_x) {
        auto in_place = [&](const Rows &r) { return r.p == d_x && r.stride == d_x_stride; };
        if (!apart(size, rdx, size, rx) || !apart(size, rdx, size, rs) || (!in_place(ro) && !apart(size, rdx, size, ro)) ||
            (!in_place(ra) && !apart(size, rdx, size, ra)) || !clear_of_own(f, mask, size, rdx))
            return ECRM_EINVAL;
    }
    if (!weights && !d_x) return ECRM_OK;

    // where d_x takes the place of what the weights' products read, it comes behind them
    const bool both = weights && d_x && (mask || d_x != d_out);
    make_plan(f, kPlanBack, N);
    if (both) {
        make_plan(f, kPlanBoth, N);
    } else {
        if (weights) make_plan(f, kPlanWeights, N);
        if (d_x) make_plan(f, kPlanInput, N);
    }
    if (!is_planned(f->plans.back) || (d_x && !is_planned(both ? f->plans.both : f->plans.input)) ||
        (weights && !both && !is_planned(f->plans.weights)))
        return ECRM_EINVAL;

    void *h = f->work + f->off_h, *dg = f->work + f->off_dg, *du = f->work + f->off_du;
    a.part = (float *)(f->work + f->off_part);
    const void *e = d_out;                // without the factor
    uint64_t e_stride = d_out_stride;
    float scale = 1.0f;
    if (mask) {
        e = f->work + f->off_e;
        e_stride = f->e_pitch;
        scale = a.mask.factor;
        a.mask.factor = 1.0f;
        launch_dropout(a.mask, d_out, d_out_stride, nullptr, 0, (void *)e, e_stride, type, n, D, st);
    }
    a.activation = f->cfg.activation;
    a.accumulate = accumulate ? 1u : 0u;
    a.wide = weight_type != type ? 1u : 0u;
    a.arrived = (uint32_t *)(f->work + f->off_arrived);
    a.clear = both ? counters_of(f->plans.both) : 0u;
    if (!both && weights) a.clear = counters_of(f->plans.weights);
    if (!both && d_x && counters_of(f->plans.input) > a.clear) a.clear = counters_of(f->plans.input);
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        a.p[0] = product(e, e_stride, f->down, f->down_stride, N, F, D);
        a.p[0].in = saved;
        a.p[0].out = dg;
        a.p[0].out2 = du;
        a.p[0].out3 = h;
        a.p[0].out_stride = f->pitch;
        a.p[0].scale = scale;
        BlockLaunch<T>::back(a, f->plans.back, (uint32_t)f->cus, st);
        Product w[3], in;
        w[0] = product(dg, f->pitch, x, x_stride, F, D, N);
        w[0].out = d_gate;
        w[1] = product(du, f->pitch, x, x_stride, F, D, N);
        w[1].out = d_up;
        w[2] = product(e, e_stride, h, f->pitch, D, F, N);
        w[2].out = d_down;
        w[2].scale = scale;
        w[0].out_stride = w[1].out_stride = D;
        w[2].out_stride = F;
        for (Product &p : w) p.kind = kWeights;
        in = product(dg, f->pitch, f->gate_weights, f->gate_stride, N, D, F);
        in.a.p[1] = du;
        in.b.p[1] = f->up;
        in.b.stride[1] = f->up_stride;
        in.in = add;
        in.in_stride = add_stride;
        in.out = d_x;
        in.out_stride = d_x_stride;
        in.kind = kInput;
        if (weights && !both) BlockLaunch<T>::gradients(a, w, nullptr, f->plans.weights, st);
        if (d_x) BlockLaunch<T>::gradients(a, both ? w : nullptr, &in, both ? f->plans.both : f->plans.input, st);
    });
    return launched();
}

}  // extern "C"

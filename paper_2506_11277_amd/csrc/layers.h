// Host-side declarations of the feed-forward operators: what ozimmu_layers.h's entry points call, per element type.
#pragma once
#include "layers_dev.h"

namespace oz {

inline size_t element_bytes(int type) { return type == OZIMMU_F32 ? 4 : 2; }

constexpr int kFewTokens = 16;             // columns few_tokens_kernel takes
ProductPlan plan_product(int np, int nq, int nk, int type, bool k_rows, bool direct);
int plan_pair(const Product &x, const ProductPlan &xp, const Product &w, const ProductPlan &wp, int type, bool bias);
inline size_t product_partial_bytes(int np, int nq, const ProductPlan &p)
{
    return p.splits > 1 ? (size_t)p.splits * nq * ((np + 7) / 8 * 8) * 4 : 0;
}
hipError_t launch_product_bf16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st);
hipError_t launch_pair_bf16(const Product &dx, const Product &dw, const BiasGrad &db, int tile, hipStream_t st);
hipError_t launch_product_f16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st);
hipError_t launch_pair_f16(const Product &dx, const Product &dw, const BiasGrad &db, int tile, hipStream_t st);
hipError_t launch_product_f32(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st);
hipError_t launch_pair_f32(const Product &dx, const Product &dw, const BiasGrad &db, int tile, hipStream_t st);

// rows of `cols` entries, `ld` apart, to rows `ldto` apart (a multiple of 8), zeros behind them (pad.hip)
struct PadCopy {
    const void *from;
    void *to;
    long long rows;
    int cols, ld, ldto;
};
struct PadCopies {
    PadCopy c[2];                          // rows = 0: none
};
hipError_t launch_pad(const PadCopies &a, int type, hipStream_t st);

// dz = dy * act'(pre) and the sums of its columns (grad.hip)
// Tokens a work-group sums: 64, fewer where that leaves fewer than 1024 work-groups, at least two a wavefront, more where
// the grid would grow beyond its limit.
inline int grad_rows(int tokens, int n_out)
{
    const long long strips = (n_out + 511) / 512;
    int rows = 64;
    while (rows > 8 && strips * ((tokens + rows - 1) / rows) < 1024) rows /= 2;
    while ((tokens + rows - 1) / rows > 65535) rows *= 2;
    return rows;
}
struct GradInput {
    const void *dy, *pre;                  // pre may be null (no activation)
    void *dz;                              // null: only the sums
    float *sums;                           // [ceil(tokens / rows)][n_out], null: none
    int lddy, ldpre, lddz, tokens, n_out, rows, act, wide;
};
hipError_t launch_grad_input(const GradInput &g, int type, hipStream_t st);
hipError_t launch_bias_grad(const BiasGrad &b, int type, hipStream_t st);

// a mixture-of-experts layer on a few tokens (moe.hip)
struct MoeArgs {
    const void *x, *router, *w_in, *w_out;
    int *chosen;
    float *gates;
    void *h, *y;                           // h: [tokens * top_k] rows of the hidden layer, ldh apart (16 bits: and again, what the first ones leave)
    float *parts;                          // [moe_out_parts][tokens][width]
    int ldx, ldh, ldy, tokens, width, hidden, experts, top_k, normalise;
};
// Parts of the experts' steps that the last launch divides among work-groups of the same features: as many as fill the 256
// compute units, of at least 8 steps a wavefront (8 tokens, 64 experts of 2048 x 1024: 57 us in one part).
inline int moe_out_parts(int tokens, int width, int hidden, int experts, int top_k, size_t size)
{
    const long long can = (long long)tokens * top_k < experts ? (long long)tokens * top_k : experts;
    const long long items = can * ((hidden * (long long)size + 127) / 128), groups = (width + 15) / 16;
    int parts = 1;
    while (parts < 8 && groups * parts * 2 <= 256 && items / (parts * 2) >= 8 * 16) parts *= 2;
    return parts;
}
hipError_t launch_moe(const MoeArgs &a, int type, hipStream_t st);

}  // namespace oz

// Host-side declarations of the feed-forward operators: what ozimmu_layers.h's entry points call, per element type.
#pragma once
#include "layers_dev.h"

namespace oz {

constexpr int kType8 = 8;                  // operands in 8 bits (whole numbers), beside the types that callers name
inline size_t element_bytes(int type) { return type == OZIMMU_F32 ? 4 : type == kType8 ? 1 : 2; }

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
// operands in 8 bits, results of the named type
hipError_t launch_product8_bf16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st);
hipError_t launch_product8_f16(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st);
hipError_t launch_product8_f32(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st);

// rows of `cols` entries, `ld` apart, to rows `ldto` apart (a multiple of 8, in 8 bits of 16), zeros behind them (pad.hip)
struct PadCopy {
    const void *from;
    void *to;
    long long rows;
    int cols, ld, ldto;
    const float *scale;                    // of the rows, where `from` is held in 8 bits; else null
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
    int lddy, ldpre, lddz, tokens, n_out, rows, act;
    const float *pre_scale;                // of the rows of pre, where it is held in 8 bits; else null
    // scales whose m goes into dz, null: none; 1 / m of the tokens and of the output features
    const float *x_scale, *w_scale;
    float *x_inverse, *w_inverse;
};
// (neither dz nor sums: the copies alone)
hipError_t launch_grad_input(const GradInput &g, const PadCopies &copies, int type, hipStream_t st);
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

// the root-mean-square norm of rows, and rows to 8 bits (norm.hip)
struct NormArgs {
    const void *x, *residual, *weight;     // residual and weight may be null
    void *total, *y;                       // either may be null
    int8_t *codes;                         // null: no rows in 8 bits
    float *scale;                          // null: nor scales
    int ldx, ldr, ldt, ldy, ldc, rows, width;
    float eps;
    int norm;                              // 0: to 8 bits as they are
};
hipError_t launch_norm(const NormArgs &a, int type, hipStream_t st);

// its gradients (norm_grad.hip)
struct NormGradArgs {
    const void *dy, *h, *weight, *add;     // weight and add may be null
    void *dx, *dw;                         // either may be null
    float *sums;                           // [parts][width], null without dw
    float *factors;                        // [rows][2] where the rows are not kept in registers and there is a dw, else null
    int lddy, ldh, ldadd, lddx, rows, width;
    float eps;
};
// Parts of the rows whose sums of dw are formed apart, and how: rows in registers, dw beside them, or in a pass by columns, `group` rows a part.
// (Up to 512 parts, 1024 of rows of 1025 to 1536 values where there are many, and more where a part would have more than 1024 rows.  With 1024 8192 x 8192 bf16 takes 111 us instead of 106, 2048 x 8192 42 instead of 35, for their sums alone; with two rows a part
// at least 512 x 4096 11.4 instead of 12.7, but 64 x 4096 7.4 instead of 6.7 and 1531 x 1001 f16 12.9 instead of 11.9.)
struct NormGradPlan {
    bool in_registers;
    int parts, group;
};
inline NormGradPlan plan_norm_grad(int rows, int width)
{
    // (and no more than 1024 rows one behind the other in a sum of 32 bits)
    NormGradPlan p{width <= 16384, 0, 64};
    // (rows of 1025 to 1536 values leave many of 256 threads without one, and more work-groups make up for it: 30000 x 1500 bf16 77 us with 1024 parts, 94
    // with 512, but 16384 x 2048 53.5 with 1024, 48.5 with 512)
    constexpr int kMostRows = 1024;
    const int most = width > 1024 && width <= 1536 && rows >= 8192 ? 1024 : 512;
    if (p.in_registers) {
        const int each = width <= 1024 ? 4 : 1, groups = (int)((rows + each - 1LL) / each), least = (int)((groups + kMostRows - 1LL) / kMostRows);
        p.parts = groups < most ? groups : least > most ? least : most;
    } else {
        const int even = (int)((rows + most - 1LL) / most);
        if (even > p.group) p.group = even < 4 * kMostRows ? even : 4 * kMostRows;
        p.parts = (int)((rows + p.group - 1LL) / p.group);
    }
    return p;
}
hipError_t launch_norm_grad(const NormGradArgs &a, int type, hipStream_t st);

}  // namespace oz

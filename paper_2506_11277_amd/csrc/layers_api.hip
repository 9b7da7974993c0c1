// extern "C" boundary of the feed-forward operators (ozimmu_layers.h): argument checks, plans, kernel sequencing.
#include "layers.h"

namespace oz {

// Tile and number of parts of the contraction.  A launch takes as many rounds as its work-groups need on 256 compute
// units; a round of tiles costs their entries times the steps over the rate that tile reaches where it fills the chip.
ProductPlan plan_product(int np, int nq, int nk, int type, bool k_rows)
{
    const int ke = type == OZIMMU_F32 ? 32 : 64;
    const int all = (nk + ke - 1) / ke;
    if (k_rows && nq <= kFewTokens) {
        // work-groups of 16 features; the contraction is divided where they leave most compute units without one
        const int groups = (np + 15) / 16;
        int s = 1;
        while (s < 16 && groups * s * 2 <= 256 && all / (2 * s) >= 16) s *= 2;
        const int steps = (all + s - 1) / s;
        return ProductPlan{kTileFew, steps > 0 ? (all + steps - 1) / steps : 1, steps, false};
    }
    static const int edge[3] = {256, 128, 64};
    static const double rate[3] = {1.0, 0.8, 0.5};
    ProductPlan best{2, 1, all, false};
    double least = 0;
    for (int t = type == OZIMMU_F32 ? 1 : 0; t < 3; ++t) {
        const double tiles = (double)((np + edge[t] - 1) / edge[t]) * ((nq + edge[t] - 1) / edge[t]);
        for (int s = 1; s <= 16 && (s == 1 || all / s >= 4); s *= 2) {
            const double groups = tiles * s;
            const double rounds = __builtin_ceil(groups / 256);
            const int steps = (all + s - 1) / s;
            // in units of a step of a 64 x 64 tile; each work-group has a start and an end, a join reads the parts
            const double cost = rounds * (edge[t] / 64) * (edge[t] / 64) / rate[t] * (steps + 4) + (s > 1 ? 24 + (double)np * nq * s / (64 * 64 * 64) : 0);
            if (least == 0 || cost < least) {
                least = cost;
                best = ProductPlan{t, (all + steps - 1) / (steps > 0 ? steps : 1), steps, false};
                if (best.splits < 1) best.splits = 1;
            }
        }
    }
    return best;
}

}  // namespace oz

using namespace oz;

namespace {

inline bool bad_type(int type) { return type != OZIMMU_BF16 && type != OZIMMU_F16 && type != OZIMMU_F32; }

// a matrix of `rows` rows of `cols` entries, `ld` apart
inline bool bad_rows(int rows, int cols, const void *p, int ld, size_t size)
{
    if (rows < 0 || cols < 0 || ld < (cols > 1 ? cols : 1)) return true;
    if (rows == 0 || cols == 0) return false;
    return p == nullptr || (uintptr_t)p % size != 0;
}

inline size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

inline bool on16(const void *p, int ld, size_t size) { return ((uintptr_t)p | (size_t)ld * size) % 16 == 0; }

// whether an operand can be copied to LDS 16 bytes at a time (`along`: its entries along the contiguous side)
inline bool direct_operand(const void *p, int ld, int along, size_t size)
{
    return on16(p, ld, size) && (size_t)along * size % 16 == 0 && 256ull * (unsigned)ld * size < (1ull << 32);
}

hipError_t launch_product(Product a, ProductPlan plan, int type, float *partial, hipStream_t st)
{
    const size_t size = element_bytes(type);
    Epilogue &e = a.e;
    if (e.np == 0 || e.nq == 0) return hipSuccess;
    plan.direct = a.nk > 0 && direct_operand(a.P, a.ldp, a.p_k_rows ? a.nk : e.np, size) && direct_operand(a.Q, a.ldq, a.q_k_rows ? a.nk : e.nq, size);
    e.wide = on16(e.out, e.ldo, size) && (!e.bias || (uintptr_t)e.bias % 16 == 0) && (!e.residual || on16(e.residual, e.ldr, size)) &&
             (!e.pre || on16(e.pre, e.ldpre, size));
    return type == OZIMMU_BF16  ? launch_product_bf16(a, plan, partial, st)
           : type == OZIMMU_F16 ? launch_product_f16(a, plan, partial, st)
                                : launch_product_f32(a, plan, partial, st);
}

// parts of the workspace of ozimmu_linear_grad
struct GradWorkspace {
    size_t dz, sums, partial, total;
    int lddz;
};
GradWorkspace grad_workspace(int tokens, int n_in, int n_out, int type, int activation)
{
    GradWorkspace w{};
    w.lddz = (n_out + 7) & ~7;
    w.sums = activation == OZIMMU_ACT_NONE ? 0 : padded((size_t)tokens * w.lddz * element_bytes(type));
    w.partial = w.sums + padded((size_t)((tokens + grad_rows(tokens, n_out) - 1) / grad_rows(tokens, n_out)) * n_out * 4);
    const size_t dx = product_partial_bytes(n_in, tokens, plan_product(n_in, tokens, n_out, type, false));
    const size_t dw = product_partial_bytes(n_in, n_out, plan_product(n_in, n_out, tokens, type, false));
    w.total = w.partial + padded(dx > dw ? dx : dw);
    return w;
}

inline bool bad_workspace(const void *p, size_t have, size_t want)
{
    return want > 0 && (p == nullptr || have < want || (uintptr_t)p % 256 != 0);
}

}  // namespace

extern "C" {

size_t ozimmu_linear_workspace_bytes(int tokens, int n_in, int n_out, int type)
{
    if (tokens < 0 || n_in < 0 || n_out < 0 || bad_type(type)) return 0;
    return product_partial_bytes(n_out, tokens, plan_product(n_out, tokens, n_in, type, true));
}

int ozimmu_linear(int tokens, int n_in, int n_out, int type, const void *x, int ldx, const void *w, int ldw, const void *bias,
                  const void *residual, int ldr, int activation, void *pre, int ldpre, void *y, int ldy, void *workspace,
                  size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU) return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, n_in, x, ldx, size) || bad_rows(n_out, n_in, w, ldw, size) || bad_rows(tokens, n_out, y, ldy, size)) return OZIMMU_BAD_ARG;
    if ((uintptr_t)bias % size || (residual && bad_rows(tokens, n_out, residual, ldr, size)) || (pre && bad_rows(tokens, n_out, pre, ldpre, size)))
        return OZIMMU_BAD_ARG;
    const ProductPlan plan = plan_product(n_out, tokens, n_in, type, true);
    if (bad_workspace(workspace, workspace_bytes, product_partial_bytes(n_out, tokens, plan))) return OZIMMU_BAD_ARG;
    Product a{};
    a.P = w;
    a.ldp = ldw;
    a.p_k_rows = true;
    a.Q = x;
    a.ldq = ldx;
    a.q_k_rows = true;
    a.nk = n_in;
    a.e = Epilogue{bias, residual, pre, y, ldr, ldpre, ldy, n_out, tokens, activation, 0};
    return launch_product(a, plan, type, (float *)workspace, (hipStream_t)stream) == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

size_t ozimmu_linear_grad_workspace_bytes(int tokens, int n_in, int n_out, int type, int activation)
{
    if (tokens < 0 || n_in < 0 || n_out < 0 || bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU) return 0;
    return grad_workspace(tokens, n_in, n_out, type, activation).total;
}

int ozimmu_linear_grad(int tokens, int n_in, int n_out, int type, const void *dy, int lddy, const void *x, int ldx, const void *w,
                       int ldw, const void *pre, int ldpre, int activation, void *dx, int lddx, void *dw, int lddw, void *db,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU || tokens < 0 || n_in < 0 || n_out < 0) return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, n_out, dy, lddy, size) || (activation && bad_rows(tokens, n_out, pre, ldpre, size)) || (uintptr_t)db % size) return OZIMMU_BAD_ARG;
    if (dx && (bad_rows(tokens, n_in, dx, lddx, size) || bad_rows(n_out, n_in, w, ldw, size))) return OZIMMU_BAD_ARG;
    if (dw && (bad_rows(n_out, n_in, dw, lddw, size) || bad_rows(tokens, n_in, x, ldx, size))) return OZIMMU_BAD_ARG;
    const GradWorkspace ws = grad_workspace(tokens, n_in, n_out, type, activation);
    if (bad_workspace(workspace, workspace_bytes, ws.total)) return OZIMMU_BAD_ARG;
    if (n_out == 0 && !dx) return OZIMMU_OK;
    const hipStream_t st = (hipStream_t)stream;
    char *const base = (char *)workspace;

    const void *dz = dy;
    int lddz = lddy;
    if (n_out > 0 && (db || (activation && (dx || dw)))) {
        GradInput g{};
        g.dy = dy;
        g.pre = activation ? pre : nullptr;
        g.dz = activation && (dx || dw) ? base + ws.dz : nullptr;
        g.db = db;
        g.sums = (float *)(base + ws.sums);
        g.lddy = lddy;
        g.ldpre = ldpre;
        g.lddz = ws.lddz;
        g.tokens = tokens;
        g.n_out = n_out;
        g.rows = grad_rows(tokens, n_out);
        g.act = activation;
        g.wide = on16(dy, lddy, size) && (!activation || on16(pre, ldpre, size));
        if (launch_grad_input(g, type, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    }
    if (activation) {
        dz = base + ws.dz;
        lddz = ws.lddz;
    }
    float *partial = (float *)(base + ws.partial);
    Product a{};
    if (dx) {
        a.P = w;
        a.ldp = ldw;
        a.Q = dz;
        a.ldq = lddz;
        a.q_k_rows = true;
        a.nk = n_out;
        a.e = Epilogue{nullptr, nullptr, nullptr, dx, 0, 0, lddx, n_in, tokens, OZIMMU_ACT_NONE, 0};
        if (launch_product(a, plan_product(n_in, tokens, n_out, type, false), type, partial, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    }
    if (dw) {
        a.P = x;
        a.ldp = ldx;
        a.Q = dz;
        a.ldq = lddz;
        a.q_k_rows = false;
        a.nk = tokens;
        a.e = Epilogue{nullptr, nullptr, nullptr, dw, 0, 0, lddw, n_in, n_out, OZIMMU_ACT_NONE, 0};
        if (launch_product(a, plan_product(n_in, n_out, tokens, type, false), type, partial, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    }
    return OZIMMU_OK;
}

size_t ozimmu_moe_workspace_bytes(int tokens, int width, int hidden, int experts, int top_k, int type)
{
    if (tokens < 0 || tokens > OZIMMU_MOE_TOKENS || width < 0 || hidden < 0 || experts < 1 || experts > OZIMMU_MOE_EXPERTS || top_k < 1 ||
        top_k > experts || top_k > OZIMMU_MOE_TOP_K || bad_type(type))
        return 0;
    return padded((size_t)tokens * top_k * ((hidden + 7) & ~7) * element_bytes(type));
}

int ozimmu_moe(int tokens, int width, int hidden, int experts, int top_k, int type, int normalise, const void *x, int ldx,
               const void *router, const void *w_in, const void *w_out, int32_t *chosen, float *gates, void *y, int ldy,
               void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || tokens < 0 || tokens > OZIMMU_MOE_TOKENS || width < 0 || hidden < 0 || hidden > 0x3fffffff || experts < 1 ||
        experts > OZIMMU_MOE_EXPERTS || top_k < 1 || top_k > experts || top_k > OZIMMU_MOE_TOP_K)
        return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, width, x, ldx, size) || bad_rows(tokens, width, y, ldy, size) || bad_rows(experts, width, router, width > 1 ? width : 1, size) ||
        bad_rows(2 * hidden, width, w_in, width > 1 ? width : 1, size) || bad_rows(width, hidden, w_out, hidden > 1 ? hidden : 1, size))
        return OZIMMU_BAD_ARG;
    if (tokens > 0 && (!chosen || !gates || (uintptr_t)chosen % 4 || (uintptr_t)gates % 4)) return OZIMMU_BAD_ARG;
    if (bad_workspace(workspace, workspace_bytes, ozimmu_moe_workspace_bytes(tokens, width, hidden, experts, top_k, type))) return OZIMMU_BAD_ARG;
    if (tokens == 0) return OZIMMU_OK;
    const MoeArgs a{x, router, w_in, w_out, chosen, gates, workspace, y, ldx, (hidden + 7) & ~7, ldy, tokens, width, hidden, experts, top_k, normalise != 0};
    return launch_moe(a, type, (hipStream_t)stream) == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

}  // extern "C"

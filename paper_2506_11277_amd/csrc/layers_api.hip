// extern "C" boundary of the feed-forward operators (ozimmu_layers.h): argument checks, plans, kernel sequencing.
#include "../../include/ozimmu_bench.h"
#include "layers.h"

namespace oz {

// Tile and number of parts of the contraction, by the time that each would take.  A launch takes as many rounds as its
// work-groups need on 256 compute units (two 64 x 64 tiles fit one, but share its LDS, which bounds them, so that they take turns in effect).  Times in
// us, measured on 128^3 ... 8192^3: of a launch, of a tile's start and epilogue, of a step of 64 (32 bits: 32) of k:
//   256 x 256   2 + rounds (10 + 1.53 steps)   4096^3 bf16: 112, against 149 with 128 x 128
//   128 x 128   3 + rounds (3 + 0.53 steps)    2048^3 bf16: 22, against 28 with 64 x 64 and 50 with 256 x 256
//    64 x 64    3 + rounds (0.7 + 0.20 steps)  200 x 2048 x 2048: 9.7, against 18 with 128 x 128
// (binary32: 2.07 and 0.52 a step); a join of parts 3.5 and its reads and writes at 8 TB/s.
static const struct {
    int edge;
    double launch, tile, step16, step32;
} kShapes[3] = {{256, 2, 10, 1.53, 0}, {128, 3, 3, 0.53, 2.07}, {64, 3, 0.7, 0.20, 0.52}};
static double tiles_of(int t, int np, int nq)
{
    const int e = kShapes[t].edge;
    return (double)((np + e - 1) / e) * ((nq + e - 1) / e);
}
// (operands that go to LDS through registers: a step takes two to three times as long in 16 bits, a fifth longer in 32)
// (a step of 128 bytes of k takes operands of 8 bits as long as those of 16, with twice the k)
static int step_entries(int type) { return 128 / (int)element_bytes(type); }
static double tile_us(int t, int steps, int type, bool direct = true) { return kShapes[t].tile + steps * (type == OZIMMU_F32 ? kShapes[t].step32 : kShapes[t].step16) * (direct ? 1 : type == OZIMMU_F32 ? 1.2 : 2.5); }

ProductPlan plan_product(int np, int nq, int nk, int type, bool k_rows, bool direct)
{
    const int ke = step_entries(type);
    const int all = (nk + ke - 1) / ke;
    if (k_rows && nq <= kFewTokens) {
        // work-groups of 16 features; the contraction is divided where they leave most compute units without one
        const int groups = (np + 15) / 16;
        int s = 1;
        while (s < 16 && groups * s * 2 <= 256 && all / (2 * s) >= 16) s *= 2;
        const int steps = (all + s - 1) / s;
        return ProductPlan{kTileFew, steps > 0 ? (all + steps - 1) / steps : 1, steps, direct, 0};
    }
    ProductPlan best{kTile64, 1, all, direct, 1e300};
    for (int t = type == OZIMMU_F32 || !direct ? kTile128 : kTile256; t <= kTile64; ++t)
        for (int s = 1; s <= 16 && (s == 1 || all / s >= 4); s *= 2) {
            const int steps = (all + s - 1) / s;
            const double us = kShapes[t].launch + __builtin_ceil(tiles_of(t, np, nq) * s / 256) * tile_us(t, steps, type, direct) +
                              (s > 1 ? 3.5 + (double)np * nq * s * 8 / 8e6 : 0);
            if (us < best.us) best = ProductPlan{t, steps > 0 ? (all + steps - 1) / steps : 1, steps, direct, us};
        }
    return best;
}

// The tile with which two products take one launch, or -1 where two launches are sooner done (2 us for the second one, 3 for
// the bias gradient's).
int plan_pair(const Product &x, const ProductPlan &xp, const Product &w, const ProductPlan &wp, int type, bool bias)
{
    const int ke = step_entries(type);
    int best = -1;
    double least = xp.us + wp.us + 2 + (bias ? 3 : 0);
    for (int t = kTile128; t <= kTile64; ++t) {
        const double ux = tile_us(t, (x.nk + ke - 1) / ke, type), uw = tile_us(t, (w.nk + ke - 1) / ke, type), longest = ux > uw ? ux : uw;
        const double all = (tiles_of(t, x.e.np, x.e.nq) * ux + tiles_of(t, w.e.np, w.e.nq) * uw) / 256;
        const double us = kShapes[t].launch + (all < longest / 2 ? longest : all + longest / 2);
        if (us < least) {
            least = us;
            best = t;
        }
    }
    // (32 bits: a step's matrix instructions keep a compute unit busy, and half of the units would have none: 500 x 512 x 384 10.7 us instead of 14.6)
    if (best == kTile64 && type == OZIMMU_F32 && tiles_of(kTile64, x.e.np, x.e.nq) + tiles_of(kTile64, w.e.np, w.e.nq) <= 128) return kTile32;
    return best;
}

static int edge_of(int tile) { return tile == kTileFew ? 16 : tile == kTile32 ? 32 : kShapes[tile].edge; }

}  // namespace oz

using namespace oz;

namespace {

inline bool bad_type(int type) { return type != OZIMMU_BF16 && type != OZIMMU_F16 && type != OZIMMU_F32; }

constexpr int kMostRows = (1 << 30) - 1;       // (numbers of steps and tiles are ints)

// a matrix of `rows` rows of `cols` entries, `ld` apart
inline bool bad_rows(int rows, int cols, const void *p, int ld, size_t size)
{
    if (rows < 0 || cols < 0 || rows > kMostRows || cols > kMostRows || ld < (cols > 1 ? cols : 1)) return true;
    if (rows == 0 || cols == 0) return false;
    return p == nullptr || (uintptr_t)p % size != 0;
}

inline bool bad_sizes(int a, int b, int c) { return a < 0 || b < 0 || c < 0 || a > kMostRows || b > kMostRows || c > kMostRows; }

inline size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

inline bool on16(const void *p, int ld, size_t size) { return ((uintptr_t)p | (size_t)ld * size) % 16 == 0; }

// whether an operand can be copied to LDS 16 bytes at a time (`along`: its entries along the contiguous side)
inline bool direct_operand(const void *p, int ld, int along, size_t size)
{
    return on16(p, ld, size) && (size_t)along * size % 16 == 0 && 256ull * (unsigned)ld * size < (1ull << 32);
}

// entries of a row of a copy
inline int up(int n, size_t size) { return size == 1 ? (n + 15) & ~15 : (n + 7) & ~7; }
inline int up8(int n) { return (n + 7) & ~7; }

// bytes of the copies of a product's operands (P, Q) in aligned rows
inline size_t copy_bytes(const Product &a, bool of_p, size_t size)
{
    const size_t rows = of_p ? (a.p_k_rows ? a.p_rows : a.p_nk) : (a.q_k_rows ? a.q_rows : a.q_nk);
    const int along = of_p ? (a.p_k_rows ? a.p_nk : a.p_rows) : (a.q_k_rows ? a.q_nk : a.q_rows);
    return padded(rows * up(along, size) * size);
}

// The plan of a product, and the copies that it wants first (`space`: where they go; null: there is no room, or too little).
// type: of the operands, result: of what the epilogue reads and writes, launch_us: what a launch for copies costs.
ProductPlan route_product(Product &a, int type, int result, bool k_rows, char *space, size_t space_bytes, PadCopies &copies, double launch_us = 6)
{
    const size_t size = element_bytes(type), out = element_bytes(result);
    Epilogue &e = a.e;
    e.wide = on16(e.out, e.ldo, out) && (!e.bias || (uintptr_t)e.bias % 16 == 0) && (!e.residual || on16(e.residual, e.ldr, out)) &&
             (!e.pre || on16(e.pre, e.ldpre, out)) && (uintptr_t)e.p_scale % 16 == 0;
    copies = PadCopies{};
    const bool p_fits = direct_operand(a.P, a.ldp, a.p_k_rows ? a.p_nk : a.p_rows, size), q_fits = direct_operand(a.Q, a.ldq, a.q_k_rows ? a.q_nk : a.q_rows, size);
    const ProductPlan direct = plan_product(e.np, e.nq, a.nk, type, k_rows, true);
    if (direct.tile == kTileFew || (a.nk > 0 && p_fits && q_fits)) return direct;
    const ProductPlan other = plan_product(e.np, e.nq, a.nk, type, k_rows, false);
    // (a copy whose rows are too long for direct operands is of no use)
    const int p_along = a.p_k_rows ? a.p_nk : a.p_rows, q_along = a.q_k_rows ? a.q_nk : a.q_rows;
    if (256ull * up(p_along, size) * size >= (1ull << 32) || 256ull * up(q_along, size) * size >= (1ull << 32)) return other;
    const size_t p_bytes = p_fits ? 0 : copy_bytes(a, true, size), q_bytes = q_fits ? 0 : copy_bytes(a, false, size);
    // The copies: a launch, and their bytes read and written at 4 TB/s.  Rows off 16 bytes, without and with them: 4096^3 f16 321 and
    // 128 us (aligned: 110), 1024 x 4096 x 1024 52 and 30, 1531 x 1000 x 776 17 either way, 200 x 1000 x 4000 15 and 19.
    if (a.nk == 0 || space == nullptr || space_bytes < p_bytes + q_bytes || direct.us + launch_us + 2 * (p_bytes + q_bytes) / 4e6 >= other.us) return other;
    auto copy = [&](PadCopy &c, const void *&x, int &ld, bool rows_along_k, int &rows, int &nk, char *to) {
        int &along = rows_along_k ? nk : rows;
        c = PadCopy{x, to, rows_along_k ? rows : nk, along, ld, up(along, size), nullptr};
        x = to;
        ld = along = c.ldto;
    };
    if (!p_fits) copy(copies.c[0], a.P, a.ldp, a.p_k_rows, a.p_rows, a.p_nk, space);
    if (!q_fits) copy(copies.c[1], a.Q, a.ldq, a.q_k_rows, a.q_rows, a.q_nk, space + p_bytes);
    return direct;
}

hipError_t launch_product(const Product &a, const ProductPlan &plan, int type, float *partial, hipStream_t st)
{
    if (a.e.np == 0 || a.e.nq == 0) return hipSuccess;
    return type == OZIMMU_BF16  ? launch_product_bf16(a, plan, partial, st)
           : type == OZIMMU_F16 ? launch_product_f16(a, plan, partial, st)
                                : launch_product_f32(a, plan, partial, st);
}

// partial sums of a product whichever way its operands go
inline size_t either_partial_bytes(int np, int nq, int nk, int type, bool k_rows)
{
    const size_t a = product_partial_bytes(np, nq, plan_product(np, nq, nk, type, k_rows, true)), b = product_partial_bytes(np, nq, plan_product(np, nq, nk, type, k_rows, false));
    return padded(a > b ? a : b);
}

// parts of the workspace of ozimmu_linear: partial sums, copies of x and w (where they are wanted)
struct LinearWorkspace {
    size_t copies, copies_bytes, total;
};
LinearWorkspace linear_workspace(int tokens, int n_in, int n_out, int type, bool aligned)
{
    LinearWorkspace w{};
    const size_t size = element_bytes(type);
    w.copies = either_partial_bytes(n_out, tokens, n_in, type, true);
    const ProductPlan direct = plan_product(n_out, tokens, n_in, type, true, true), other = plan_product(n_out, tokens, n_in, type, true, false);
    if ((!aligned || n_in * size % 16) && direct.tile != kTileFew && direct.us + 3 < other.us)
        w.copies_bytes = padded((size_t)tokens * up(n_in, size) * size) + padded((size_t)n_out * up(n_in, size) * size);
    w.total = w.copies + w.copies_bytes;
    return w;
}

// parts of the workspace of ozimmu_linear_grad and ozimmu_linear8_grad; x8, w8: held in 8 bits, and always copied
struct GradWorkspace {
    size_t dz, sums, inverse_x, inverse_w, partial, copies_x, copies_w, total;
    bool has_dz, has_x, has_w, split;          // split: scales go into dz and the results' rows by parts (split_scale)
    int lddz;
};
GradWorkspace grad_workspace(int tokens, int n_in, int n_out, int type, int activation, bool aligned, bool x8 = false, bool w8 = false)
{
    GradWorkspace w{};
    const size_t size = element_bytes(type);
    aligned = aligned && n_in * size % 16 == 0 && n_out * size % 16 == 0;
    w.lddz = up8(n_out);
    w.split = (x8 || w8) && size == 2;
    w.has_dz = activation != OZIMMU_ACT_NONE || !aligned || w.split;
    w.has_x = x8 || !aligned;
    w.has_w = w8 || !aligned;
    w.sums = w.has_dz ? padded((size_t)tokens * w.lddz * size) : 0;
    w.inverse_x = w.sums + padded((size_t)((tokens + grad_rows(tokens, n_out) - 1) / grad_rows(tokens, n_out)) * n_out * 4);
    w.inverse_w = w.inverse_x + (w.split && x8 ? padded((size_t)tokens * 4) : 0);
    w.partial = w.inverse_w + (w.split && w8 ? padded((size_t)n_out * 4) : 0);
    const size_t dx = either_partial_bytes(n_in, tokens, n_out, type, false), dw = either_partial_bytes(n_in, n_out, tokens, type, false);
    w.copies_x = w.partial + (dx > dw ? dx : dw);
    w.copies_w = w.copies_x + (w.has_x ? padded((size_t)tokens * up8(n_in) * size) : 0);
    w.total = w.copies_w + (w.has_w ? padded((size_t)n_out * up8(n_in) * size) : 0);
    return w;
}

inline bool bad_workspace(const void *p, size_t have, size_t want)
{
    return want > 0 && (p == nullptr || have < want || (uintptr_t)p % 256 != 0);
}

// ozimmu_linear and ozimmu_linear8, their arguments checked but for the workspace: operands of `type`, the rest of `result`
int linear(int tokens, int n_in, int n_out, int type, int result, const void *x, int ldx, const float *x_scale, const void *w, int ldw, const float *w_scale,
           const void *bias, const void *residual, int ldr, int activation, void *pre, int ldpre, void *y, int ldy, void *workspace,
           size_t workspace_bytes, void *stream)
{
    if (bad_workspace(workspace, workspace_bytes, linear_workspace(tokens, n_in, n_out, type, true).total)) return OZIMMU_BAD_ARG;
    if (tokens == 0 || n_out == 0) return OZIMMU_OK;
    const LinearWorkspace ws = linear_workspace(tokens, n_in, n_out, type, false);
    // (a workspace that is not needed may be anywhere, but copies go to 16 bytes)
    const bool room = ws.copies_bytes > 0 && workspace_bytes >= ws.total && (uintptr_t)workspace % 256 == 0;
    Product a{};
    a.P = w;
    a.ldp = ldw;
    a.p_k_rows = true;
    a.p_rows = n_out;
    a.Q = x;
    a.ldq = ldx;
    a.q_k_rows = true;
    a.q_rows = tokens;
    a.nk = a.p_nk = a.q_nk = n_in;
    a.e = Epilogue{bias, residual, pre, y, ldr, ldpre, ldy, n_out, tokens, activation, x_scale, w_scale, 0};
    PadCopies copies;
    const ProductPlan plan = route_product(a, type, result, true, room ? (char *)workspace + ws.copies : nullptr, ws.copies_bytes, copies);
    const hipStream_t st = (hipStream_t)stream;
    if (launch_pad(copies, type, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    float *const partial = (float *)workspace;
    const hipError_t e = type != kType8            ? launch_product(a, plan, type, partial, st)
                         : result == OZIMMU_BF16 ? launch_product8_bf16(a, plan, partial, st)
                         : result == OZIMMU_F16  ? launch_product8_f16(a, plan, partial, st)
                                                 : launch_product8_f32(a, plan, partial, st);
    return e == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

// ozimmu_linear_grad and ozimmu_linear8_grad: x, w and pre of `type`, or held in 8 bits where they have scales
int linear_grad(int tokens, int n_in, int n_out, int type, const void *dy, int lddy, const void *x, int ldx, const float *x_scale, const void *w, int ldw,
                const float *w_scale, const void *pre, int ldpre, const float *pre_scale, int activation, void *dx, int lddx, void *dw, int lddw,
                void *db, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU || bad_sizes(tokens, n_in, n_out)) return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, n_out, dy, lddy, size) || (activation && bad_rows(tokens, n_out, pre, ldpre, pre_scale ? 1 : size)) || (uintptr_t)db % size) return OZIMMU_BAD_ARG;
    if (dx && (bad_rows(tokens, n_in, dx, lddx, size) || bad_rows(n_out, n_in, w, ldw, w_scale ? 1 : size))) return OZIMMU_BAD_ARG;
    if (dw && (bad_rows(n_out, n_in, dw, lddw, size) || bad_rows(tokens, n_in, x, ldx, x_scale ? 1 : size))) return OZIMMU_BAD_ARG;
    const bool x8 = x_scale != nullptr, w8 = w_scale != nullptr;
    GradWorkspace ws = grad_workspace(tokens, n_in, n_out, type, activation, true, x8, w8);
    if (bad_workspace(workspace, workspace_bytes, ws.total)) return OZIMMU_BAD_ARG;
    if (n_out == 0 && !dx) return OZIMMU_OK;
    const hipStream_t st = (hipStream_t)stream;
    char *const base = (char *)workspace;
    // (dy of no activation is read as it is where it can be copied directly, or there is no room for dz)
    const bool dy_fits = direct_operand(dy, lddy, n_out, size);
    if (!dy_fits || (dx && !w8 && !direct_operand(w, ldw, n_in, size)) || (dw && !x8 && !direct_operand(x, ldx, n_in, size))) {
        const GradWorkspace wider = grad_workspace(tokens, n_in, n_out, type, activation, false, x8, w8);
        if (workspace_bytes >= wider.total) ws = wider;
    }

    // (also where only one of dx and dw is wanted: the products' operands are the same whichever is, and only the order of their sums goes by that)
    const bool split_x = ws.split && x8, split_w = ws.split && w8;
    const bool own_dz = n_out > 0 && (dx || dw) && (activation || split_x || split_w || (ws.has_dz && !dy_fits));
    const void *dz = dy;
    int lddz = lddy, dz_cols = n_out;
    const int rows = grad_rows(tokens, n_out);
    GradInput g{};
    if (n_out > 0 && (db || own_dz)) {
        g.dy = dy;
        g.pre = activation ? pre : nullptr;
        g.dz = own_dz ? base + ws.dz : nullptr;
        g.sums = db ? (float *)(base + ws.sums) : nullptr;
        g.lddy = lddy;
        g.ldpre = ldpre;
        g.lddz = ws.lddz;
        g.tokens = tokens;
        g.n_out = n_out;
        g.rows = rows;
        g.act = activation;
        g.pre_scale = activation ? pre_scale : nullptr;
        if (own_dz && split_x) {
            g.x_scale = x_scale;
            g.x_inverse = (float *)(base + ws.inverse_x);
        }
        if (own_dz && split_w) {
            g.w_scale = w_scale;
            g.w_inverse = (float *)(base + ws.inverse_w);
        }
    }
    if (own_dz) {
        dz = base + ws.dz;
        lddz = dz_cols = ws.lddz;
    }
    const BiasGrad bias{(const float *)(base + ws.sums), db, (tokens + rows - 1) / rows, n_out};
    float *partial = (float *)(base + ws.partial);
    Product x_grad{}, w_grad{};
    x_grad.P = w;
    x_grad.ldp = ldw;
    x_grad.p_rows = n_in;
    x_grad.p_nk = n_out;
    x_grad.Q = dz;
    x_grad.ldq = lddz;
    x_grad.q_k_rows = true;
    x_grad.q_rows = tokens;
    x_grad.q_nk = dz_cols;
    x_grad.nk = n_out;
    x_grad.e = Epilogue{nullptr, nullptr, nullptr, dx, 0, 0, lddx, n_in, tokens, OZIMMU_ACT_NONE, nullptr, nullptr, 0};
    w_grad.P = x;
    w_grad.ldp = ldx;
    w_grad.p_rows = n_in;
    w_grad.p_nk = tokens;
    w_grad.Q = dz;
    w_grad.ldq = lddz;
    w_grad.q_rows = dz_cols;
    w_grad.q_nk = tokens;
    w_grad.nk = tokens;
    w_grad.e = Epilogue{nullptr, nullptr, nullptr, dw, 0, 0, lddw, n_in, n_out, OZIMMU_ACT_NONE, nullptr, nullptr, 0};
    x_grad.e.q_scale = g.x_inverse;
    w_grad.e.q_scale = tokens > 0 ? g.w_inverse : nullptr;         // (which a token's launch writes)
    PadCopies x_copies{}, w_copies{}, copies{};
    ProductPlan x_plan{}, w_plan{};
    const bool form_dx = dx && tokens > 0 && n_in > 0, form_dw = dw && n_out > 0 && n_in > 0;
    // what is held in 8 bits is copied as the values it stands for
    auto expand = [&](Product &a, const float *scale, int rows_, char *to) {
        const PadCopy c{a.P, to, rows_, n_in, a.ldp, up8(n_in), scale};
        a.P = to;
        a.ldp = a.p_rows = c.ldto;
        return c;
    };
    PadCopy w_values{}, x_values{};
    if (form_dx && w8) w_values = expand(x_grad, w_scale, n_out, base + ws.copies_w);
    if (form_dw && x8) x_values = expand(w_grad, x_scale, tokens, base + ws.copies_x);
    // (what is in 8 bits has a launch, which takes other copies along: 948 x 91 -> 768 f16 38 us with w through registers, 16 with a copy)
    const double launch_us = x8 || w8 ? 0.5 : 6;
    // (of each product P alone can want a copy here: dz is the workspace's, or dy where there is no room for either)
    if (form_dx) x_plan = route_product(x_grad, type, type, false, ws.has_w && !w8 ? base + ws.copies_w : nullptr, ws.total - ws.copies_w, x_copies, launch_us);
    if (form_dw) w_plan = route_product(w_grad, type, type, false, ws.has_x && !x8 ? base + ws.copies_x : nullptr, ws.copies_w - ws.copies_x, w_copies, launch_us);
    copies.c[0] = w8 ? w_values : x_copies.c[0];
    copies.c[1] = x8 ? x_values : w_copies.c[0];
    if (launch_grad_input(g, copies, type, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    const bool both = form_dx && form_dw && n_out > 0 && tokens > 0 && x_plan.direct && w_plan.direct;
    const int pair = both ? plan_pair(x_grad, x_plan, w_grad, w_plan, type, db != nullptr) : -1;
    if (pair >= 0) {
        const hipError_t e = type == OZIMMU_BF16  ? launch_pair_bf16(x_grad, w_grad, bias, pair, st)
                             : type == OZIMMU_F16 ? launch_pair_f16(x_grad, w_grad, bias, pair, st)
                                                  : launch_pair_f32(x_grad, w_grad, bias, pair, st);
        return e == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
    }
    if (launch_bias_grad(bias, type, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    if (form_dx && launch_product(x_grad, x_plan, type, partial, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    if (form_dw && launch_product(w_grad, w_plan, type, partial, st) != hipSuccess) return OZIMMU_HIP_ERROR;
    return OZIMMU_OK;
}

}  // namespace

extern "C" {

size_t ozimmu_linear_workspace_bytes(int tokens, int n_in, int n_out, int type, int aligned)
{
    if (bad_sizes(tokens, n_in, n_out) || bad_type(type)) return 0;
    return linear_workspace(tokens, n_in, n_out, type, aligned != 0).total;
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
    return linear(tokens, n_in, n_out, type, type, x, ldx, nullptr, w, ldw, nullptr, bias, residual, ldr, activation, pre, ldpre, y, ldy, workspace, workspace_bytes, stream);
}

size_t ozimmu_linear8_workspace_bytes(int tokens, int n_in, int n_out, int aligned)
{
    if (bad_sizes(tokens, n_in, n_out) || n_in > OZIMMU_LINEAR8_IN) return 0;
    return linear_workspace(tokens, n_in, n_out, kType8, aligned != 0).total;
}

int ozimmu_linear8(int tokens, int n_in, int n_out, int type, const int8_t *x, int ldx, const float *x_scale, const int8_t *w, int ldw,
                   const float *w_scale, const void *bias, const void *residual, int ldr, int activation, void *pre, int ldpre, void *y,
                   int ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU || n_in > OZIMMU_LINEAR8_IN) return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, n_in, x, ldx, 1) || bad_rows(n_out, n_in, w, ldw, 1) || bad_rows(tokens, n_out, y, ldy, size)) return OZIMMU_BAD_ARG;
    if ((uintptr_t)bias % size || (residual && bad_rows(tokens, n_out, residual, ldr, size)) || (pre && bad_rows(tokens, n_out, pre, ldpre, size)))
        return OZIMMU_BAD_ARG;
    if ((tokens > 0 && !x_scale) || (n_out > 0 && !w_scale) || (uintptr_t)x_scale % 4 || (uintptr_t)w_scale % 4) return OZIMMU_BAD_ARG;
    return linear(tokens, n_in, n_out, kType8, type, x, ldx, x_scale, w, ldw, w_scale, bias, residual, ldr, activation, pre, ldpre, y, ldy, workspace,
                  workspace_bytes, stream);
}

int ozimmu_debug_linear_tile(int which, int tokens, int n_in, int n_out, int type, int aligned, int *parts)
{
    if (which < 0 || which > 3 || bad_sizes(tokens, n_in, n_out) || (bad_type(type) && !(which == 0 && type == kType8))) return OZIMMU_BAD_ARG;
    const int np = which == 0 ? n_out : n_in, nq = which == 2 ? n_out : tokens, nk = which == 0 ? n_in : which == 1 ? n_out : tokens;
    const ProductPlan plan = plan_product(np, nq, nk, type, which == 0, aligned != 0);
    if (parts) *parts = which == 3 ? 1 : plan.splits;
    if (which < 3) return edge_of(plan.tile);
    Product dx{}, dw{};
    dx.nk = n_out;
    dx.e.np = dw.e.np = n_in;
    dx.e.nq = dw.nk = tokens;
    dw.e.nq = n_out;
    const int tile = plan_pair(dx, plan_product(n_in, tokens, n_out, type, false, true), dw, plan_product(n_in, n_out, tokens, type, false, true), type, true);
    return tile < 0 ? 0 : edge_of(tile);
}

size_t ozimmu_linear_grad_workspace_bytes(int tokens, int n_in, int n_out, int type, int activation, int aligned)
{
    if (bad_sizes(tokens, n_in, n_out) || bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU) return 0;
    return grad_workspace(tokens, n_in, n_out, type, activation, aligned != 0).total;
}

int ozimmu_linear_grad(int tokens, int n_in, int n_out, int type, const void *dy, int lddy, const void *x, int ldx, const void *w,
                       int ldw, const void *pre, int ldpre, int activation, void *dx, int lddx, void *dw, int lddw, void *db,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    return linear_grad(tokens, n_in, n_out, type, dy, lddy, x, ldx, nullptr, w, ldw, nullptr, pre, ldpre, nullptr, activation, dx, lddx, dw, lddw, db,
                       workspace, workspace_bytes, stream);
}

size_t ozimmu_linear8_grad_workspace_bytes(int tokens, int n_in, int n_out, int type, int activation, int aligned, int x8, int w8)
{
    if (bad_sizes(tokens, n_in, n_out) || bad_type(type) || activation < OZIMMU_ACT_NONE || activation > OZIMMU_ACT_SILU) return 0;
    return grad_workspace(tokens, n_in, n_out, type, activation, aligned != 0, x8 != 0, w8 != 0).total;
}

int ozimmu_linear8_grad(int tokens, int n_in, int n_out, int type, const void *dy, int lddy, const void *x, int ldx, const float *x_scale,
                        const void *w, int ldw, const float *w_scale, const void *pre, int ldpre, const float *pre_scale, int activation,
                        void *dx, int lddx, void *dw, int lddw, void *db, void *workspace, size_t workspace_bytes, void *stream)
{
    if ((uintptr_t)x_scale % 4 || (uintptr_t)w_scale % 4 || (uintptr_t)pre_scale % 4) return OZIMMU_BAD_ARG;
    return linear_grad(tokens, n_in, n_out, type, dy, lddy, x, ldx, x_scale, w, ldw, w_scale, pre, ldpre, pre_scale, activation, dx, lddx, dw, lddw, db,
                       workspace, workspace_bytes, stream);
}

}  // extern "C"

namespace {
constexpr int kMostFeatures = 1 << 24;         // (all chosen experts' steps are counted in an int)

// parts of the workspace of ozimmu_moe
struct MoeWorkspace {
    size_t parts, total;
    int ldh;
};
MoeWorkspace moe_workspace(int tokens, int width, int hidden, int experts, int top_k, int type)
{
    MoeWorkspace w{};
    const size_t size = element_bytes(type);
    const int parts = moe_out_parts(tokens, width, hidden, experts, top_k, size);
    w.ldh = (hidden + 7) & ~7;
    w.parts = padded((size_t)tokens * top_k * w.ldh * 4);           // (one number of 32 bits or two of 16)
    w.total = w.parts + (parts > 1 ? padded((size_t)parts * tokens * width * 4) : 0);
    return w;
}
}  // namespace

extern "C" {

size_t ozimmu_moe_workspace_bytes(int tokens, int width, int hidden, int experts, int top_k, int type)
{
    if (tokens < 0 || tokens > OZIMMU_MOE_TOKENS || width < 0 || width > kMostFeatures || hidden < 0 || hidden > kMostFeatures || experts < 1 ||
        experts > OZIMMU_MOE_EXPERTS || top_k < 1 || top_k > experts || top_k > OZIMMU_MOE_TOP_K || bad_type(type))
        return 0;
    return moe_workspace(tokens, width, hidden, experts, top_k, type).total;
}

int ozimmu_moe(int tokens, int width, int hidden, int experts, int top_k, int type, int normalise, const void *x, int ldx,
               const void *router, const void *w_in, const void *w_out, int32_t *chosen, float *gates, void *y, int ldy,
               void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || tokens < 0 || tokens > OZIMMU_MOE_TOKENS || width < 0 || width > kMostFeatures || hidden < 0 || hidden > kMostFeatures || experts < 1 ||
        experts > OZIMMU_MOE_EXPERTS || top_k < 1 || top_k > experts || top_k > OZIMMU_MOE_TOP_K)
        return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, width, x, ldx, size) || bad_rows(tokens, width, y, ldy, size) || bad_rows(experts, width, router, width > 1 ? width : 1, size) ||
        bad_rows(2 * hidden, width, w_in, width > 1 ? width : 1, size) || bad_rows(width, hidden, w_out, hidden > 1 ? hidden : 1, size))
        return OZIMMU_BAD_ARG;
    if (tokens > 0 && (!chosen || !gates || (uintptr_t)chosen % 4 || (uintptr_t)gates % 4)) return OZIMMU_BAD_ARG;
    const MoeWorkspace ws = moe_workspace(tokens, width, hidden, experts, top_k, type);
    if (bad_workspace(workspace, workspace_bytes, ws.total)) return OZIMMU_BAD_ARG;
    if (tokens == 0) return OZIMMU_OK;
    const MoeArgs a{x, router, w_in, w_out, chosen, gates, workspace, y, (float *)((char *)workspace + ws.parts),
                    ldx, ws.ldh, ldy, tokens, width, hidden, experts, top_k, normalise != 0};
    return launch_moe(a, type, (hipStream_t)stream) == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

}  // extern "C"

namespace {
inline bool bad_eps(double eps) { return !((float)eps > 0.0f) || !((float)eps <= 3.402823466e38f); }

// parts of the workspace of ozimmu_rms_norm_grad
struct NormGradWorkspace {
    size_t factors, total;
};
NormGradWorkspace norm_grad_workspace(int tokens, int width)
{
    const NormGradPlan p = plan_norm_grad(tokens, width);
    NormGradWorkspace w{};
    w.factors = padded((size_t)p.parts * width * 4);
    w.total = w.factors + (p.in_registers ? 0 : padded((size_t)tokens * 8));
    return w;
}
}  // namespace

extern "C" {

int ozimmu_rms_norm(int tokens, int width, int type, const void *x, int ldx, const void *residual, int ldr, const void *weight, double eps,
                    void *total, int ldt, void *y, int ldy, int8_t *codes, int ldc, float *scale, void *stream)
{
    if (bad_type(type) || bad_sizes(tokens, width, 0) || bad_eps(eps)) return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, width, x, ldx, size) || (residual && bad_rows(tokens, width, residual, ldr, size)) || (uintptr_t)weight % size ||
        (total && bad_rows(tokens, width, total, ldt, size)) || (y && bad_rows(tokens, width, y, ldy, size)) ||
        (codes && bad_rows(tokens, width, codes, ldc, 1)) || (codes && tokens > 0 && !scale) || (scale && !codes && tokens > 0 && width > 0) || (uintptr_t)scale % 4)
        return OZIMMU_BAD_ARG;
    if (!total && !y && !scale) return OZIMMU_OK;
    const NormArgs a{x, residual, weight, total, y, codes, scale, ldx, ldr, ldt, ldy, ldc, tokens, width, (float)eps, 1};
    return launch_norm(a, type, (hipStream_t)stream) == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

int ozimmu_quantise(int rows, int cols, int type, const void *x, int ldx, int8_t *codes, int ldc, float *scale, void *stream)
{
    if (bad_type(type) || bad_sizes(rows, cols, 0)) return OZIMMU_BAD_ARG;
    if (bad_rows(rows, cols, x, ldx, element_bytes(type)) || bad_rows(rows, cols, codes, ldc, 1) || (rows > 0 && !scale) || (uintptr_t)scale % 4) return OZIMMU_BAD_ARG;
    NormArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.codes = codes;
    a.ldc = ldc;
    a.scale = scale;
    a.rows = rows;
    a.width = cols;
    return launch_norm(a, type, (hipStream_t)stream) == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

size_t ozimmu_rms_norm_grad_workspace_bytes(int tokens, int width)
{
    return bad_sizes(tokens, width, 0) ? 0 : norm_grad_workspace(tokens, width).total;
}

int ozimmu_rms_norm_grad(int tokens, int width, int type, const void *dy, int lddy, const void *h, int ldh, const void *weight, double eps,
                         const void *add, int ldadd, void *dx, int lddx, void *dw, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_type(type) || bad_sizes(tokens, width, 0) || bad_eps(eps)) return OZIMMU_BAD_ARG;
    const size_t size = element_bytes(type);
    if (bad_rows(tokens, width, dy, lddy, size) || bad_rows(tokens, width, h, ldh, size) || (uintptr_t)weight % size ||
        (add && bad_rows(tokens, width, add, ldadd, size)) || (dx && bad_rows(tokens, width, dx, lddx, size)) || (uintptr_t)dw % size)
        return OZIMMU_BAD_ARG;
    const NormGradWorkspace ws = norm_grad_workspace(tokens, width);
    if (dw && bad_workspace(workspace, workspace_bytes, ws.total)) return OZIMMU_BAD_ARG;
    if (width == 0 || (!dx && !dw)) return OZIMMU_OK;
    char *const base = (char *)workspace;
    const bool factors = dw && !plan_norm_grad(tokens, width).in_registers;
    const NormGradArgs a{dy, h, weight, add, dx, dw, dw ? (float *)base : nullptr, factors ? (float *)(base + ws.factors) : nullptr,
                         lddy, ldh, ldadd, lddx, tokens, width, (float)eps};
    return launch_norm_grad(a, type, (hipStream_t)stream) == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

}  // extern "C"

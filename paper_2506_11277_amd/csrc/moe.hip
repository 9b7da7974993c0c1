// A mixture-of-experts layer for a few tokens.  Bound by memory: the weights of the chosen experts, read once.
//
//   moe_route_kernel   a work-group per token: logits of all experts, the chosen ones and their gates (for one to four tokens and
//                      a small router the second kernel does that by itself)
//   moe_hidden_kernel  a work-group per 16 hidden features of an expert that some token chose: gate and up rows against
//                      the tokens that chose it, h = gate silu(a) b
//   moe_out_kernel     a work-group per 16 output features: their rows of every chosen expert against its tokens' h, all in one
//                      sum, so nothing is scattered and no atomics change an order; in two to eight parts, which
//                      moe_join_kernel adds, where the features are too few for all compute units
//
// 8 tokens, 64 experts of 2048 x 1024 bf16, 8 chosen (42 different ones): routing 9 us, hidden layer 80 (352 MB at 4.4 TB/s), output 36 to
// 40 (176 MB at 4.4 to 4.9) and 5.
//
// Which experts are chosen is known on the device only: the second launch has a work-group for each of the min(experts,
// tokens * top_k) experts that can be, which finds its expert in a bit map of the chosen ones and leaves if there is none.
#include "layers.h"
#include "stream_dev.h"

namespace oz {
namespace {

constexpr int kRouteWaves = 16, kHiddenWaves = 4, kOutWaves = 16;
constexpr int kWords = OZIMMU_MOE_EXPERTS / 32;
// The hidden layer is kept as the sum of two numbers of 16 bits (bf16: to 2^-16 of h; f16: to 2^-22 of it, but to no less than 2^-25):
// rounded to one, it alone would add as much to the result's error as the result's own rounding.  The second one's products take
// matrix instructions that wait for memory anyway.
template <class T>
constexpr int kParts = sizeof(T) == 2 ? 2 : 1;

// h's numbers: h itself, or the nearest number of 16 bits and what it leaves.  A finite h that f16 has no number for becomes a NaN for the
// matrix instructions, so that the sums show it, and 26 bits of its own for the second look that they then get: its sign and how far
// |h|'s bits are above those of 2^15, without the last five; the first number has the upper 9 of these 25 behind what makes it a
// NaN, the second one the others.
constexpr unsigned kLeastCode = 0x47000000u;                    // 2^15
__device__ __forceinline__ void put_hidden(float h, float *first, size_t) { *first = h; }
__device__ __forceinline__ void put_hidden(float h, bf16 *first, size_t second)
{
    const float most = 0x1.fep127f;                             // (bf16's largest: larger ones would be rounded to infinity)
    const bf16 b = (bf16)(fabsf(h) < __builtin_inff() ? fminf(fmaxf(h, -most), most) : h);
    first[0] = b;
    first[second] = (bf16)(fabsf(h) < __builtin_inff() ? h - (float)b : 0.0f);
}
__device__ __forceinline__ void put_hidden(float h, f16 *first, size_t second)
{
    const f16 b = (f16)h;
    unsigned short one = __builtin_bit_cast(unsigned short, b), two = 0;
    if (h != h) {
        one = 0x7e00;
    } else if (fabsf(h) < __builtin_inff()) {
        if (fabsf((float)b) < __builtin_inff()) {
            two = __builtin_bit_cast(unsigned short, (f16)(h - (float)b));
        } else {
            const unsigned bits = __float_as_uint(h), code = ((bits & 0x7fffffffu) - kLeastCode) >> 5;      // (25 bits, at least 3 << 16)
            one = (unsigned short)((bits >> 16 & 0x8000u) | 0x7e00u | code >> 16);
            two = (unsigned short)code;
        }
    }
    first[0] = __builtin_bit_cast(f16, one);
    first[second] = __builtin_bit_cast(f16, two);
}
__device__ __forceinline__ float get_hidden(float first, float) { return first; }
__device__ __forceinline__ float get_hidden(bf16 first, bf16 second) { return (float)first + (float)second; }
__device__ __forceinline__ float get_hidden(f16 first, f16 second)
{
    const unsigned one = __builtin_bit_cast(unsigned short, first), two = __builtin_bit_cast(unsigned short, second);
    if ((one & 0x7e00u) == 0x7e00u && (one & 0x1ffu) != 0)
        return __uint_as_float((one & 0x8000u) << 16 | ((((one & 0x1ffu) << 16 | two) << 5 | 16) + kLeastCode));
    return (float)first + (float)second;
}
constexpr int kRouteHere = 64;                                  // choices that fit the second kernel's own routing

// bit map of the experts that the `n` choices name
__device__ __forceinline__ void mark_chosen(unsigned *map, const int *chosen, int n)
{
    for (int i = threadIdx.x; i < kWords; i += blockDim.x) map[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += blockDim.x) atomicOr(&map[chosen[i] >> 5], 1u << (chosen[i] & 31));
    __syncthreads();
}

// how many experts below e are marked
__device__ __forceinline__ int marked_before(const unsigned *map, int e)
{
    int n = __popc(map[e >> 5] & ((1u << (e & 31)) - 1));
    for (int i = 0; i < e >> 5; ++i) n += __popc(map[i]);
    return n;
}

// a > b, a NaN above everything, for a at a later place than b if `later` (ties go to the earlier one)
__device__ __forceinline__ bool before(float a, float b, bool later)
{
    const bool an = a != a, bn = b != b;
    if (an || bn) return an && (!bn || !later);
    return later ? a > b : a >= b;
}

// The choice of token t by a work-group of WAVES wavefronts: its experts in ascending order, and their gates.
struct RouteSpace {
    float logits[OZIMMU_MOE_EXPERTS], share[OZIMMU_MOE_EXPERTS];
    unsigned map[kWords];
    float total;
};
template <class T, int WAVES>
__device__ __forceinline__ void route_token(const MoeArgs &a, int t, RouteSpace &space, int *chosen, float *gates)
{
    constexpr int E = Chunk<T>::E;
    typedef typename Chunk<T>::V V;
    float *logits = space.logits, *share = space.share;
    unsigned *map = space.map;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const T *x = (const T *)a.x + (size_t)t * a.ldx;
    for (int i = threadIdx.x; i < kWords; i += blockDim.x) map[i] = 0;
    // four experts of a wavefront at a time, all of whose loads of four steps are issued before the first product
    const int whole = a.width / (64 * E) * (64 * E);
    for (int e0 = wave; e0 < a.experts; e0 += 4 * WAVES) {
        const T *r[4];
        float s[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = e0 + i * WAVES;
            r[i] = (const T *)a.router + (size_t)(e < a.experts ? e : e0) * a.width;
        }
        auto products = [&](v4u xc, const v4u (&rc)[4]) {
            const V xv = __builtin_bit_cast(V, xc);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const V rv = __builtin_bit_cast(V, rc[i]);
#pragma unroll
                for (int c = 0; c < E; ++c) s[i] = __builtin_fmaf((float)xv[c], (float)rv[c], s[i]);
            }
        };
        int k = lane * E;
        for (; k + 3 * 64 * E < whole; k += 4 * 64 * E) {
            v4u xc[4], rc[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                __builtin_memcpy(&xc[u], x + k + u * 64 * E, 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) __builtin_memcpy(&rc[u][i], r[i] + k + u * 64 * E, 16);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 4; ++u) products(xc[u], rc[u]);
        }
        for (; k < whole; k += 64 * E) {
            v4u xc, rc[4];
            __builtin_memcpy(&xc, x + k, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) __builtin_memcpy(&rc[i], r[i] + k, 16);
            products(xc, rc);
        }
        if (whole + lane * E < a.width) {
            const int k = whole + lane * E, n = a.width - k;
            const v4u xc = load_chunk(x + k, n);
            const v4u rc[4] = {load_chunk(r[0] + k, n), load_chunk(r[1] + k, n), load_chunk(r[2] + k, n), load_chunk(r[3] + k, n)};
            products(xc, rc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int d = 32; d; d >>= 1) s[i] += __shfl_xor(s[i], d);
            if (lane == 0 && e0 + i * WAVES < a.experts) logits[e0 + i * WAVES] = s[i];
        }
    }
    __syncthreads();
    // an expert is chosen if fewer than top_k come before it: 16 lanes count for it
    for (int e = threadIdx.x >> 4; e < (a.experts + 3) / 4 * 4; e += 4 * WAVES) {
        const bool there = e < a.experts;
        const float l = there ? logits[e] : 0.0f;
        int rank = 0;
        for (int o = threadIdx.x & 15; there && o < a.experts; o += 16) rank += o != e && before(logits[o], l, o > e);
#pragma unroll
        for (int d = 8; d; d >>= 1) rank += __shfl_xor(rank, d);
        if (there && (threadIdx.x & 15) == 0 && rank < a.top_k) atomicOr(&map[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
    // the sum of the exponentials, by one wavefront
    if (wave == 0) {
        float top = -__builtin_inff();
        for (int e = lane; e < a.experts; e += 64) top = fmaxf(top, logits[e]);
#pragma unroll
        for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
        float sum = 0.0f;
        for (int e = lane; e < a.experts; e += 64) {
            const float v = expf(logits[e] - top);
            share[e] = v;
            if (!a.normalise || (map[e >> 5] >> (e & 31) & 1)) sum += v;
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) space.total = sum;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x) {
        if (!(map[e >> 5] >> (e & 31) & 1)) continue;
        const int place = marked_before(map, e);
        chosen[place] = e;
        gates[place] = share[e] / space.total;
    }
}

template <class T>
__global__ __launch_bounds__(64 * kRouteWaves) void moe_route_kernel(MoeArgs a)
{
    __shared__ RouteSpace space;
    const int t = blockIdx.x;
    route_token<T, kRouteWaves>(a, t, space, a.chosen + t * a.top_k, a.gates + t * a.top_k);
}

// ROUTE: every work-group finds the choices for itself (the first one writes them down)
template <class T, bool ROUTE>
__global__ __launch_bounds__(64 * kHiddenWaves) void moe_hidden_kernel(MoeArgs a)
{
    constexpr int KE = 8 * Chunk<T>::E;
    __shared__ unsigned map[kWords];
    __shared__ int own_chosen[ROUTE ? kRouteHere : 1];
    __shared__ float own_gates[ROUTE ? kRouteHere : 1];
    __shared__ typename std::conditional<ROUTE, RouteSpace, int>::type space;
    __shared__ int choices[OZIMMU_MOE_TOKENS];                 // of the tokens that chose this expert: token * top_k + place
    __shared__ int count;
    __shared__ __attribute__((aligned(16))) float sums[kHiddenWaves][2][16 * kStreamLd];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int all = a.tokens * a.top_k;
    const int *chosen = ROUTE ? own_chosen : a.chosen;
    const float *gates = ROUTE ? own_gates : a.gates;
    if constexpr (ROUTE) {
        for (int t = 0; t < a.tokens; ++t) {
            route_token<T, kHiddenWaves>(a, t, space, own_chosen + t * a.top_k, own_gates + t * a.top_k);
            __syncthreads();
        }
        if (blockIdx.x == 0 && blockIdx.y == 0)
            for (int i = threadIdx.x; i < all; i += blockDim.x) {
                a.chosen[i] = own_chosen[i];
                a.gates[i] = own_gates[i];
            }
    }
    mark_chosen(map, chosen, all);
    int expert = -1;
    for (int i = 0, left = blockIdx.y; i < kWords; ++i) {      // the blockIdx.y-th bit that is set
        unsigned m = map[i];
        const int n = __popc(m);
        if (left >= n) {
            left -= n;
            continue;
        }
        for (; left > 0; --left) m &= m - 1;
        expert = i * 32 + __builtin_ctz(m);
        break;
    }
    if (expert < 0) return;
    if (wave == 0) {                                           // its tokens in their order: a lane each
        int mine = -1;
        if (lane < a.tokens)
            for (int i = 0; i < a.top_k; ++i)
                if (chosen[lane * a.top_k + i] == expert) mine = lane * a.top_k + i;
        const unsigned long long who = __ballot(mine >= 0);
        if (mine >= 0) choices[__popcll(who & ((1ull << lane) - 1))] = mine;
        if (lane == 0) count = __popcll(who);
    }
    __syncthreads();
    const int f0 = blockIdx.x * 16, row = f0 + (lane & 15) < a.hidden ? f0 + (lane & 15) : a.hidden - 1;
    const T *const base = (const T *)a.w_in + (size_t)expert * 2 * a.hidden * a.width;
    const T *const w[2] = {base + (size_t)row * a.width, base + ((size_t)a.hidden + row) * a.width};
    const int steps = (a.width + KE - 1) / KE;
    for (int c0 = 0; c0 < count; c0 += 16) {
        const bool on[1] = {c0 + (lane & 15) < count};
        const T *const x[1] = {(const T *)a.x + (size_t)(choices[on[0] ? c0 + (lane & 15) : 0] / a.top_k) * a.ldx};
        v4f acc[2][1] = {{v4f{0, 0, 0, 0}}, {v4f{0, 0, 0, 0}}};
        stream_products<T, 2, 1, 4>(acc, w, x, on, wave, steps, kHiddenWaves, a.width, lane);
        put_sums(sums[wave][0], acc[0][0], lane);
        put_sums(sums[wave][1], acc[1][0], lane);
        __syncthreads();
        const int i = threadIdx.x;                             // 16 tokens x 16 features
        const int q = i >> 4, f = i & 15;
        if (i < 256 && c0 + q < count && f0 + f < a.hidden) {
            float g = 0.0f, u = 0.0f;
#pragma unroll
            for (int s = 0; s < kHiddenWaves; ++s) {
                g += sums[s][0][q * kStreamLd + f];
                u += sums[s][1][q * kStreamLd + f];
            }
            const int choice = choices[c0 + q];
            const float h = gates[choice] * activate<T>(OZIMMU_ACT_SILU, g) * u;
            put_hidden(h, (T *)a.h + (size_t)choice * a.ldh + f0 + f, (size_t)all * a.ldh);
        }
        __syncthreads();
    }
}

template <class T, int NX>
__global__ __launch_bounds__(64 * kOutWaves) void moe_out_kernel(MoeArgs a)
{
    constexpr int E = Chunk<T>::E, KE = 8 * E, H = kParts<T>, U = NX == 1 ? (H == 2 ? 3 : 4) : NX == 2 ? 2 : H == 2 ? 1 : 2;
    constexpr int kNone = 255;
    __shared__ unsigned map[kWords];
    __shared__ int experts[OZIMMU_MOE_EXPERTS];                                // the chosen ones
    __shared__ uint8_t places[OZIMMU_MOE_EXPERTS * 16 * NX];                   // [chosen expert][token]: its place among the token's, or kNone
    __shared__ __attribute__((aligned(16))) float sums[kOutWaves][NX][16 * kStreamLd];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int all = a.tokens * a.top_k, can = all < a.experts ? all : a.experts;
    for (int i = threadIdx.x; i < can * 16 * NX / 4; i += blockDim.x) ((unsigned *)places)[i] = ~0u;
    mark_chosen(map, a.chosen, all);
    for (int e = threadIdx.x; e < a.experts; e += blockDim.x)
        if (map[e >> 5] >> (e & 31) & 1) experts[marked_before(map, e)] = e;
    for (int i = threadIdx.x; i < all; i += blockDim.x) {
        const int t = i / a.top_k;
        places[marked_before(map, a.chosen[i]) * 16 * NX + t] = (uint8_t)(i - t * a.top_k);
    }
    int chosen = 0;
    for (int i = 0; i < kWords; ++i) chosen += __popc(map[i]);
    __syncthreads();

    const int p0 = blockIdx.x * 16, row = p0 + (lane & 15) < a.width ? p0 + (lane & 15) : a.width - 1, g = (lane >> 4) * E;
    v4f acc[NX];
#pragma unroll
    for (int j = 0; j < NX; ++j) acc[j] = v4f{0, 0, 0, 0};
    // The steps of all chosen experts, one after the other, are dealt to the wavefronts in turn; U steps' loads, of as many
    // experts as it may be, are issued before the first of their products.
    const int steps = (a.hidden + KE - 1) / KE, items = chosen * steps;
    const size_t second = (size_t)all * a.ldh;                                 // from h's first numbers to its second ones
    const int part = (items + gridDim.y - 1) / gridDim.y, begin = blockIdx.y * part, end = begin + part < items ? begin + part : items;
    for (int first = begin + wave; first < end; first += U * kOutWaves) {
        v4u w[U][2], h[U][2][NX][H];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int item = first + u * kOutWaves;
            const bool there = item < end;
            const int slot = there ? item / steps : 0, k0 = (there ? item - slot * steps : 0) * KE + g;
            const T *wr = (const T *)a.w_out + ((size_t)experts[slot] * a.width + row) * a.hidden;
            const T *hr[NX];
            bool on[NX];
#pragma unroll
            for (int j = 0; j < NX; ++j) {
                const int t = 16 * j + (lane & 15), place = places[slot * 16 * NX + t];
                on[j] = there && place != kNone;
                hr[j] = (const T *)a.h + (size_t)(on[j] ? t * a.top_k + place : 0) * a.ldh;
            }
            if (there && k0 - g + KE <= a.hidden) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    __builtin_memcpy(&w[u][s], wr + k0 + s * 4 * E, 16);
#pragma unroll
                    for (int j = 0; j < NX; ++j) {
#pragma unroll
                        for (int o = 0; o < H; ++o) {
                            h[u][s][j][o] = v4u{0, 0, 0, 0};
                            if (on[j]) __builtin_memcpy(&h[u][s][j][o], hr[j] + o * second + k0 + s * 4 * E, 16);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int k = k0 + s * 4 * E, n = there ? a.hidden - k : 0;
                    w[u][s] = load_chunk(wr + k, n);
#pragma unroll
                    for (int j = 0; j < NX; ++j)
#pragma unroll
                        for (int o = 0; o < H; ++o) h[u][s][j][o] = load_chunk(hr[j] + o * second + k, on[j] ? n : 0);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int o = 0; o < H; ++o)
#pragma unroll
                    for (int j = 0; j < NX; ++j) acc[j] = mma(w[u][s], h[u][s][j][o], acc[j], T{});
    }
    static_assert(NX * 256 <= 64 * kOutWaves, "an entry a lane");
    const int q = threadIdx.x >> 4, p = threadIdx.x & 15;
    const bool mine = q < 16 * NX && q < a.tokens && p0 + p < a.width;
    auto entry = [&]() __attribute__((always_inline)) {                        // this lane's, of the wavefronts' sums
        __syncthreads();
        float v = 0.0f;
        if (mine)
#pragma unroll
            for (int s = 0; s < kOutWaves; ++s) v += sums[s][q >> 4][(q & 15) * kStreamLd + p];
        return v;
    };
    const auto finite = [](float x) { return fabsf(x) < __builtin_inff(); };
#pragma unroll
    for (int j = 0; j < NX; ++j) put_sums(sums[wave][j], acc[j], lane);
    float v = entry();
    // Infinities and NaN.  A token that did not choose an expert has zeros for its h, and an infinite weight times 0, or times h's two
    // numbers of unlike signs, is a NaN, and so are values of h beyond f16; so where a sum of 16 tokens is not finite, the steps are gone over again in two ways: as before, but
    // of a step a token keeps the sum only if it chose the expert (the same bits as if the others' weights were finite), and
    // with weights and h as numbers of 32 bits.  The second is taken where the first is not finite either.  (8 tokens, 64 experts of 2048 x
    // 1024, a NaN or a large h in every work-group's sums: the launch 100 to 110 us instead of 40.)
    const int again = __syncthreads_or(mine && !finite(v)) ? NX : 0;
#pragma nounroll
    for (int j = 0; j < again; ++j) {
        const bool odd = mine && q >> 4 == j && !finite(v);
        if (!__syncthreads_or(odd)) continue;
        // (a lane's own numbers once more: kept over the loop above, they cost it registers that it spills)
        int own = threadIdx.x & 63;
        asm volatile("" : "+v"(own));
        const int t = 16 * j + (own & 15), f = p0 + (own & 15) < a.width ? p0 + (own & 15) : a.width - 1;
        v4f same = {0, 0, 0, 0}, wide = {0, 0, 0, 0};
#pragma nounroll
        for (int item = begin + wave; item < end; item += kOutWaves) {
            const int slot = item / steps, k0 = (item - slot * steps) * KE + (own >> 4) * E, place = places[slot * 16 * NX + t];
            const bool on = place != kNone;
            const T *wr = (const T *)a.w_out + ((size_t)experts[slot] * a.width + f) * a.hidden;
            const T *hr = (const T *)a.h + (size_t)(on ? t * a.top_k + place : 0) * a.ldh;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                typedef typename Chunk<T>::V V;
                const int k = k0 + s * 4 * E, n = a.hidden - k;
                const v4u w = load_chunk(wr + k, n);
                v4u h[H];
                v4f sum = wide;
#pragma unroll
                for (int o = 0; o < H; ++o) h[o] = load_chunk(hr + o * second + k, on ? n : 0);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x = get_hidden(__builtin_bit_cast(V, h[0])[e], __builtin_bit_cast(V, h[H - 1])[e]);
                    sum = __builtin_amdgcn_mfma_f32_16x16x4f32((float)__builtin_bit_cast(V, w)[e], x, sum, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) wide[i] = on ? sum[i] : wide[i];
#pragma unroll
                for (int o = 0; o < H; ++o) {
                    sum = mma(w, h[o], same, T{});
#pragma unroll
                    for (int i = 0; i < 4; ++i) same[i] = on ? sum[i] : same[i];
                }
            }
        }
        put_sums(sums[wave][j], same, own);
        const float first = entry();
        __syncthreads();
        put_sums(sums[wave][j], wide, own);
        const float other = entry();
        if (odd) v = finite(first) ? first : other;
    }
    if (!mine) return;
    if (gridDim.y == 1) ((T *)a.y)[(size_t)q * a.ldy + p0 + p] = (T)v;
    else a.parts[((size_t)blockIdx.y * a.tokens + q) * a.width + p0 + p] = v;
}

// the parts' sums, in their order
template <class T>
__global__ __launch_bounds__(256) void moe_join_kernel(MoeArgs a, int parts)
{
    const size_t all = (size_t)a.tokens * a.width, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    float v = 0.0f;
    for (int y = 0; y < parts; ++y) v += a.parts[y * all + i];
    ((T *)a.y)[i / a.width * a.ldy + i % a.width] = (T)v;
}

template <class T>
hipError_t launch(const MoeArgs &a, hipStream_t st)
{
    const int can = a.tokens * a.top_k < a.experts ? a.tokens * a.top_k : a.experts;
    const dim3 hidden((a.hidden + 15) / 16, can);
    // Where the router is small enough for every work-group of the second kernel to read it from the caches (16 MB in all take
    // about 2 us), its launch is saved: one token, 16 experts of 1024 x 704: 21 us in three launches, 16 in two.
    const double read = (double)hidden.x * hidden.y * a.tokens * a.experts * a.width * sizeof(T);
    const bool here = a.hidden > 0 && a.tokens <= 4 && a.tokens * a.top_k <= kRouteHere && read <= 16e6;
    if (!here) {
        moe_route_kernel<T><<<a.tokens, 64 * kRouteWaves, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.hidden > 0) {
        if (here) moe_hidden_kernel<T, true><<<hidden, 64 * kHiddenWaves, 0, st>>>(a);
        else moe_hidden_kernel<T, false><<<hidden, 64 * kHiddenWaves, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const int groups = (a.width + 15) / 16;
    if (groups == 0) return hipSuccess;
    const dim3 out(groups, moe_out_parts(a.tokens, a.width, a.hidden, a.experts, a.top_k, sizeof(T)));
    if (a.tokens <= 16) moe_out_kernel<T, 1><<<out, 64 * kOutWaves, 0, st>>>(a);
    else if (a.tokens <= 32) moe_out_kernel<T, 2><<<out, 64 * kOutWaves, 0, st>>>(a);
    else moe_out_kernel<T, 4><<<out, 64 * kOutWaves, 0, st>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (out.y > 1) {
        moe_join_kernel<T><<<(unsigned)(((size_t)a.tokens * a.width + 255) / 256), 256, 0, st>>>(a, (int)out.y);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_moe(const MoeArgs &a, int type, hipStream_t st)
{
    return type == OZIMMU_BF16 ? launch<bf16>(a, st) : type == OZIMMU_F16 ? launch<f16>(a, st) : launch<float>(a, st);
}

}  // namespace oz

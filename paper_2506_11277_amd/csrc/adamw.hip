// One AdamW step over many tensors, moments in 32 bits or in 8.
//
//   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
//   p = (1 - lr wd) p - lr / (1 - beta1^t)  m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Bound by memory: every value is read and written once.  A launch takes up to kTensors tensors whose addresses are kernel
// arguments (no table in memory to copy or to keep), cut into chunks of whole blocks of 256 values; a wavefront has one or
// two blocks at a time, four or eight consecutive values a lane.
//
// 8 bits: blocks of 256 values share a scale, and m and sqrt(v) are held as e4m3 times scale (the root halves the range of
// exponents that v needs; a block's largest value maps to 448).  Half a wavefront has the whole block, so its maximum takes five
// exchanges between lanes.  Values are rounded up or down at random, with the probability that makes the
// mean right: 0.999 v + 0.001 g^2 moves v by less than half a unit of its last place, so that rounding to nearest would
// leave it where it is for ever.  The random word is a hash of the place, the step and the caller's seed.  A root that is not 0 is
// not rounded to 0, which would leave eps alone below an m that is still there.
//
// What the states keep is rounded as written, operation by operation (no fused multiply-add, a rounded root), so that the same step
// gives the same codes whatever the compiler makes of it; the parameter's quotient is the instruction's reciprocal, a unit
// off in a step a thousandth of p.
// Measured: 143 million values, bf16 with 8 bits, 1.44 GB: 300 us; 57 million, float with a bf16 copy, 1.58 GB: 312 us (a copy
// at 5.1 TB/s: 282 and 310).  The first in four values a lane, with the library's root and division: 355 us, bound by arithmetic.
#include "layers.h"

namespace oz {
namespace {

constexpr int kBlock = 256;                      // values that share a scale in 8 bits
constexpr int kTensors = 48;                     // 48 * 80 + 56 bytes of arguments
constexpr int kChunks = 0xffffff;                // work-groups of a launch: fewer than 2^32 work-items

struct Tensor {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    long long n;
    long long block0;                            // number of its first block among all tensors of the call
    int chunk0;                                  // its first chunk (work-group) in the launch
    int flags;                                   // copy type
};
enum { kCopyF16 = 1 };

struct Args {
    Tensor t[kTensors];
    int tensors, per_chunk;                      // blocks of a chunk, even
    float b1, c1, b2, c2, eps, rate, correction, keep;
    unsigned word0;
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

// a lane's values: together at any alignment of their type, or the n that are there, the others 0
template <class T, int kEach>
__device__ __forceinline__ void get(const T *p, int n, float (&v)[kEach])
{
    if (n >= kEach) {
        T x[kEach];
        __builtin_memcpy(x, p, sizeof(x));
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}
template <class T, int kEach>
__device__ __forceinline__ void put(T *p, int n, const float (&v)[kEach])
{
    if (n >= kEach) {
        T x[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) x[i] = (T)v[i];
        __builtin_memcpy(p, x, sizeof(x));
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

constexpr int kEach = 8;                         // values of a lane where states have 8 bits

__device__ __forceinline__ v2u get_codes(const uint8_t *p, int n)
{
    v2u c = {0, 0};
    if (n >= kEach) {
        __builtin_memcpy(&c, p, 8);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i < n) c[i >> 2] |= (unsigned)p[i] << (8 * (i & 3));
    }
    return c;
}
__device__ __forceinline__ void put_codes(uint8_t *p, int n, v2u c)
{
    if (n >= kEach) {
        __builtin_memcpy(p, &c, 8);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i < n) p[i] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ void decode(v2u c, float scale, float (&v)[kEach])
{
    typedef float v2f __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], true);
        v[4 * h] = a[0] * scale;
        v[4 * h + 1] = a[1] * scale;
        v[4 * h + 2] = b[0] * scale;
        v[4 * h + 3] = b[1] * scale;
    }
}

// the words of a lane's places from `at` on, a multiple of 8 (so that they share the upper half)
__device__ __forceinline__ void words_of(unsigned long long at, unsigned word0, unsigned (&w)[kEach])
{
    const unsigned first = ((unsigned)at + (unsigned)(at >> 32) * 0x6a09e667u) * 0x9e3779b1u + word0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        unsigned h = first + i * 0x9e3779b1u;
        h = (h ^ (h >> 15)) * 0x6a09e667u;
        h = (h ^ (h >> 13)) * 0xbb67ae85u;
        w[i] = h ^ (h >> 16);
    }
}

// Square roots.  The instruction is a unit off at times and takes no subnormal numbers: where a wavefront has values below 2^-96,
// all are scaled.  ROUNDED: r is the root rounded to nearest if r (r - ulp) < x <= r (r + ulp), else a neighbour is (Tuckerman's test: Agarwal,
// Cooley, Gustavson, Shearer, Slishman, Tuckerman, "New scalar and vector elementary functions for the IBM System/370", 1986);
// the sign of either difference is exact in a fused multiply-add (0, infinities and NaN stay as they are).
template <bool ROUNDED, int N>
__device__ __forceinline__ void roots_of(const float (&v)[N], float (&root)[N])
{
    auto root_of = [](float x) {
        const float r = __builtin_amdgcn_sqrtf(x);
        if constexpr (!ROUNDED) return r;
        const float below = __uint_as_float(__float_as_uint(r) - 1), above = __uint_as_float(__float_as_uint(r) + 1);
        const float e = __builtin_fmaf(-below, r, x), f = __builtin_fmaf(-above, r, x);
        const float s = e <= 0.0f ? below : r;
        return f > 0.0f ? above : s;
    };
    float least = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) least = fminf(least, v[i]);
    if (__builtin_expect(__ballot(least < 0x1p-96f) != 0, 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool tiny = v[i] < 0x1p-96f;
            const float r = root_of(tiny ? v[i] * 0x1p96f : v[i]);
            root[i] = tiny ? r * 0x1p-48f : r;
        }
        asm volatile("");                            // (a branch, not a selection for each)
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) root[i] = root_of(v[i]);
    }
}

// the largest of a block's values, in each of its 32 lanes: among 16 by exchanges inside the vector unit, the last one through LDS's crossbar
__device__ __forceinline__ unsigned lanes_max(unsigned x)
{
    auto with = [&](unsigned o) { x = o > x ? o : x; };
    with(__builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true));         // lane ^ 1
    with(__builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true));         // lane ^ 2
    with(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true));        // 7 - lane within 8
    with(__builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true));        // 15 - lane within 16
    with(__builtin_amdgcn_ds_swizzle(x, 0x401f));                    // lane ^ 16
    return x;
}

// A block's moments in 8 bits: |x| 448 / top, rounded up where the 20 bits below e4m3's carry with the word's.  y 2^-120 has the
// bits of e4m3 (bias 7 instead of 127) 20 places further left, also where e4m3 is subnormal, so that one multiplication,
// addition and shift make the code.  ROOT: no signs, and a value that is not 0 does not become 0.
template <bool ROOT>
__device__ __forceinline__ v2u hold_block(const float (&x)[kEach], const unsigned (&word)[kEach], float &scale)
{
    constexpr unsigned kInf = 0x7f800000u;
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const unsigned a = __float_as_uint(x[i]) & 0x7fffffffu;
        top = a > top ? a : top;
    }
    top = lanes_max(top);
    const bool odd = __ballot(top >= kInf) != 0;     // a value that is not finite: the scale goes by the others
    if (__builtin_expect(odd, 0)) {
        top = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const unsigned a = __float_as_uint(x[i]) & 0x7fffffffu;
            top = a > top && a < kInf ? a : top;
        }
        top = lanes_max(top);
        asm volatile("");
    }
    const float t = __uint_as_float(top);
    scale = t * (float)(1.0 / 448.0);
    // (below 2^-100 the quotient would overflow: such a block is held as zeros, or the smallest code)
    const float quotient = t >= 0x1p-100f ? 448.0f / t : 0.0f, factor = quotient * 0x1p-120f;
    float y[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) y[i] = fabsf(x[i]) * factor;
    // (from 2^14 on the factor nears the subnormal numbers, and from 3e11 on it would be 0: there its parts are applied one after the other)
    const bool large = t > 0x1p14f;
    if (__builtin_expect(__ballot(large) != 0, 0)) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) y[i] = large ? fabsf(x[i]) * quotient * 0x1p-120f : y[i];
        asm volatile("");
    }
    v2u codes = {0, 0};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        unsigned c = (__float_as_uint(y[i]) + word[i]) >> 20;
        c = c < 0x7e ? c : 0x7e;
        if constexpr (ROOT) {
            const unsigned least = __float_as_uint(x[i]) < 1 ? __float_as_uint(x[i]) : 1;       // 0 of 0 (roots have no sign)
            c = c > least ? c : least;
        } else {
            c |= __float_as_uint(x[i]) >> 24 & 0x80;
        }
        codes[i >> 2] |= c << (8 * (i & 3));
    }
    if (__builtin_expect(odd, 0)) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if ((__float_as_uint(x[i]) & 0x7fffffffu) >= kInf) codes[i >> 2] |= 0x7fu << (8 * (i & 3));
        asm volatile("");
    }
    return codes;
}

template <class P, class G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(const Args a)
{
    // the tensor of this chunk: the last one that starts at or before it (the same search in every lane, on scalars)
    int lo = 0, hi = a.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.t[mid].chunk0 <= (int)blockIdx.x) lo = mid;
        else hi = mid;
    }
    const Tensor &t = a.t[lo];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const long long blocks = (t.n + kBlock - 1) / kBlock;
    const long long first = (long long)((int)blockIdx.x - t.chunk0) * a.per_chunk;
    const long long last = first + a.per_chunk < blocks ? first + a.per_chunk : blocks;
    // 32 bits: four values a lane, a wavefront has a block at a time (eight: 337 us instead of 305 for 57 million values, the
    // loads of 16 bytes being 32 apart).  8 bits: eight, two blocks.
    constexpr int N = EIGHT ? kEach : 4, kLanes = kBlock / N, kBlocks = 64 / kLanes;
    for (long long some = first + kBlocks * wave; some < last; some += 4 * kBlocks) {
        // (the second block may not be there: n is then 0, and its scales are not touched)
        const long long b = some + lane / kLanes, at = b * kBlock + lane % kLanes * N;
        const int n = t.n - at < N ? (t.n > at ? (int)(t.n - at) : 0) : N;
        float p[N], g[N], m[N], v[N], root[N];
        get((const P *)t.p + at, n, p);
        get((const G *)t.g + at, n, g);
        if constexpr (EIGHT) {
            const v2u mc = get_codes((const uint8_t *)t.m + at, n), vc = get_codes((const uint8_t *)t.v + at, n);
            decode(mc, b < blocks ? t.ms[b] : 0.0f, m);
            decode(vc, b < blocks ? t.vs[b] : 0.0f, v);
        } else {
            get((const float *)t.m + at, n, m);
            get((const float *)t.v + at, n, v);
        }
        {
#pragma clang fp contract(off)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (EIGHT) v[i] = v[i] * v[i];
                m[i] = m[i] * a.b1 + g[i] * a.c1;
                v[i] = v[i] * a.b2 + (g[i] * g[i]) * a.c2;
            }
        }
        roots_of<EIGHT>(v, root);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float update = m[i] * __builtin_amdgcn_rcpf(__builtin_fmaf(root[i], a.correction, a.eps));
            p[i] = __builtin_fmaf(update, -a.rate, p[i] * a.keep);
        }
        put((P *)t.p + at, n, p);
        if (t.copy) {
            if (t.flags & kCopyF16) put((f16 *)t.copy + at, n, p);
            else put((bf16 *)t.copy + at, n, p);
        }
        if constexpr (EIGHT) {
            unsigned w[N], low[N];
            words_of((unsigned long long)t.block0 * kBlock + at, a.word0, w);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                low[i] = w[i] & 0xfffff;
                w[i] >>= 12;
            }
            float ms, vs;
            const v2u mc = hold_block<false>(m, low, ms), vc = hold_block<true>(root, w, vs);
            put_codes((uint8_t *)t.m + at, n, mc);
            put_codes((uint8_t *)t.v + at, n, vc);
            if (lane % kLanes == 0 && b < blocks) {
                t.ms[b] = ms;
                t.vs[b] = vs;
            }
        } else {
            put((float *)t.m + at, n, m);
            put((float *)t.v + at, n, v);
        }
    }
}

template <class P, class G>
hipError_t launch(const Args &a, bool eight, int chunks, hipStream_t st)
{
    if (eight) adamw_kernel<P, G, true><<<chunks, 256, 0, st>>>(a);
    else adamw_kernel<P, G, false><<<chunks, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <class P>
hipError_t launch(const Args &a, int grad_type, bool eight, int chunks, hipStream_t st)
{
    return grad_type == OZIMMU_F32   ? launch<P, float>(a, eight, chunks, st)
           : grad_type == OZIMMU_F16 ? launch<P, f16>(a, eight, chunks, st)
                                     : launch<P, bf16>(a, eight, chunks, st);
}

}  // namespace
}  // namespace oz

using namespace oz;

extern "C" int ozimmu_adamw(int tensors, const ozimmu_adamw_tensor *list, const void *const *grads, double lr, double beta1, double beta2,
                            double eps, double weight_decay, long long step, uint32_t seed, void *stream)
{
    if (tensors < 0 || (tensors > 0 && list == nullptr) || step < 1) return OZIMMU_BAD_ARG;
    if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && eps >= 0) || lr != lr || weight_decay != weight_decay) return OZIMMU_BAD_ARG;
    long long total = 0, most = 0;
    for (int i = 0; i < tensors; ++i) {
        const ozimmu_adamw_tensor &x = list[i];
        const void *g = grads ? grads[i] : x.grad;
        if (x.count < 0 || x.count > (1LL << 40)) return OZIMMU_BAD_ARG;
        for (int type : {x.param_type, x.grad_type})
            if (type != OZIMMU_BF16 && type != OZIMMU_F16 && type != OZIMMU_F32) return OZIMMU_BAD_ARG;
        if (x.state_type != OZIMMU_F32 && x.state_type != OZIMMU_E4M3) return OZIMMU_BAD_ARG;
        if (x.copy && x.copy_type != OZIMMU_BF16 && x.copy_type != OZIMMU_F16) return OZIMMU_BAD_ARG;
        if (x.count == 0) continue;
        if (!x.param || !g || !x.m || !x.v || (x.state_type == OZIMMU_E4M3 && (!x.m_scale || !x.v_scale))) return OZIMMU_BAD_ARG;
        const size_t ps = x.param_type == OZIMMU_F32 ? 4 : 2, gs = x.grad_type == OZIMMU_F32 ? 4 : 2, ss = x.state_type == OZIMMU_F32 ? 4 : 1;
        if ((uintptr_t)x.param % ps || (uintptr_t)g % gs || (uintptr_t)x.m % ss || (uintptr_t)x.v % ss || (uintptr_t)x.copy % 2 ||
            (ss == 1 && ((uintptr_t)x.m_scale % 4 || (uintptr_t)x.v_scale % 4)))
            return OZIMMU_BAD_ARG;
        total += (x.count + kBlock - 1) / kBlock;
        most = x.count > most ? x.count : most;
    }
    Args a{};
    a.b1 = (float)beta1;
    a.c1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2;
    a.c2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.rate = (float)(lr / (1.0 - __builtin_pow(beta1, (double)step)));
    a.correction = (float)(1.0 / __builtin_sqrt(1.0 - __builtin_pow(beta2, (double)step)));
    a.keep = (float)(1.0 - lr * weight_decay);
    a.word0 = seed + (uint32_t)step * 0xbb67ae85u;
    a.per_chunk = total > 16 * 4096 ? 16 : 8;       // blocks of a work-group: 2 or 4 (8 bits: 1 or 2) rounds of its wavefronts
    while (most > (long long)kChunks * kBlock * a.per_chunk) a.per_chunk *= 2;
    const hipStream_t st = (hipStream_t)stream;

    long long block0 = 0, chunks = 0;
    int kind[3] = {-1, -1, -1};
    auto flush = [&]() -> hipError_t {
        if (a.tensors == 0) return hipSuccess;
        const bool eight = kind[2] == OZIMMU_E4M3;
        const hipError_t e = kind[0] == OZIMMU_F32   ? launch<float>(a, kind[1], eight, (int)chunks, st)
                             : kind[0] == OZIMMU_F16 ? launch<f16>(a, kind[1], eight, (int)chunks, st)
                                                     : launch<bf16>(a, kind[1], eight, (int)chunks, st);
        a.tensors = 0;
        chunks = 0;
        return e;
    };
    for (int i = 0; i < tensors; ++i) {
        const ozimmu_adamw_tensor &x = list[i];
        if (x.count == 0) continue;
        const void *g = grads ? grads[i] : x.grad;
        const long long blocks = (x.count + kBlock - 1) / kBlock, need = (blocks + a.per_chunk - 1) / a.per_chunk;
        if (a.tensors == kTensors || chunks + need > kChunks || kind[0] != x.param_type || kind[1] != x.grad_type || kind[2] != x.state_type) {
            if (flush() != hipSuccess) return OZIMMU_HIP_ERROR;
            kind[0] = x.param_type;
            kind[1] = x.grad_type;
            kind[2] = x.state_type;
        }
        a.t[a.tensors++] = Tensor{x.param, g, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.count, block0, (int)chunks,
                                  x.copy && x.copy_type == OZIMMU_F16 ? kCopyF16 : 0};
        block0 += blocks;
        chunks += need;
    }
    return flush() == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

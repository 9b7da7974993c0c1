// One AdamW step over many tensors, moments in 32 bits or in 8.
//
//   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
//   p = (1 - lr wd) p - lr / (1 - beta1^t)  m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Bound by memory: every value is read and written once.  A launch takes up to kTensors tensors whose addresses are kernel
// arguments (no table in memory to copy or to keep), cut into chunks of whole blocks of 256 values; a wavefront has a block at
// a time, four consecutive values a lane.
//
// 8 bits: blocks of 256 values share a scale, and m and sqrt(v) are held as e4m3 times scale (the root halves the range of
// exponents that v needs; a block's largest value maps to 448).  A wavefront has the whole block, so its maximum takes six
// exchanges between lanes and no LDS.  Values are rounded up or down at random, with the probability that makes the
// mean right: 0.999 v + 0.001 g^2 moves v by less than half a unit of its last place, so that rounding to nearest would
// leave it where it is for ever.  The random word is a hash of the place, the step and the caller's seed.  A root that is not 0 is
// not rounded to 0, which would leave eps alone below an m that is still there.
//
// Every operation is rounded by itself (no fused multiply-add), so that the 8-bit codes are those of the formulas
// whatever the compiler makes of them.
#include "layers.h"

namespace oz {
namespace {

constexpr int kBlock = 256;
constexpr int kTensors = 48;                     // 48 * 80 + 56 bytes of arguments

struct Tensor {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    long long n;
    long long block0;                            // number of its first block among all tensors of the call
    int chunk0;                                  // its first chunk (work-group) in the launch
    int flags;                                   // kWide, copy type
};
enum { kWide = 1, kCopyF16 = 2 };

struct Args {
    Tensor t[kTensors];
    int tensors, per_chunk;                      // blocks of a chunk
    float b1, c1, b2, c2, eps, rate, correction, keep;
    unsigned word0;
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

template <class T>
__device__ __forceinline__ void get4(const T *p, int n, bool wide, float (&v)[4])
{
    if (wide && n >= 4) {
        load_row(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void put4(T *p, int n, bool wide, const float (&v)[4])
{
    if (wide && n >= 4) {
        store_row(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

__device__ __forceinline__ unsigned get_codes(const uint8_t *p, int n, bool wide)
{
    if (wide && n >= 4) return *(const unsigned *)p;
    unsigned c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) c |= (unsigned)p[i] << (8 * i);
    return c;
}
__device__ __forceinline__ void put_codes(uint8_t *p, int n, bool wide, unsigned c)
{
    if (wide && n >= 4) {
        *(unsigned *)p = c;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (uint8_t)(c >> (8 * i));
    }
}
__device__ __forceinline__ void decode(unsigned c, float scale, float (&v)[4])
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
    v[0] = a[0] * scale;
    v[1] = a[1] * scale;
    v[2] = b[0] * scale;
    v[3] = b[1] * scale;
}

__device__ __forceinline__ unsigned word_of(unsigned long long at, unsigned word0)
{
    unsigned h = ((unsigned)at + (unsigned)(at >> 32) * 0x6a09e667u) * 0x9e3779b1u + word0;
    h = (h ^ (h >> 15)) * 0x6a09e667u;
    h = (h ^ (h >> 13)) * 0xbb67ae85u;
    return h ^ (h >> 16);
}

// the largest finite magnitude of a block, in every lane
__device__ __forceinline__ float block_max(const float (&x)[4])
{
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = fabsf(x[i]);
        top = a < __builtin_inff() ? fmaxf(top, a) : top;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    return top;
}

// |x| as e4m3 of 448 / top, rounded up where the 20 bits below carry with the word's.  y 2^-120 has the bits of e4m3 (bias 7
// instead of 127) 20 places further left, also where e4m3 is subnormal.
__device__ __forceinline__ unsigned hold(float x, float inverse, unsigned word)
{
    const float a = fabsf(x);
    if (!(a < __builtin_inff())) return 0x7f;                           // NaN
    const float y = fminf(a * inverse, 448.0f) * 0x1p-120f;
    const unsigned c = (__float_as_uint(y) + word) >> 20;
    return c < 0x7e ? c : 0x7e;
}

template <class P, class G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(const Args a)
{
#pragma clang fp contract(off)
    // the tensor of this chunk: the last one that starts at or before it (the same search in every lane, on scalars)
    int lo = 0, hi = a.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.t[mid].chunk0 <= (int)blockIdx.x) lo = mid;
        else hi = mid;
    }
    const Tensor &t = a.t[lo];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const bool wide = t.flags & kWide;
    const long long blocks = (t.n + kBlock - 1) / kBlock;
    const long long first = (long long)((int)blockIdx.x - t.chunk0) * a.per_chunk;
    const long long last = first + a.per_chunk < blocks ? first + a.per_chunk : blocks;
#pragma unroll 2
    for (long long b = first + wave; b < last; b += 4) {
        const long long at = b * kBlock + lane * 4;
        const int n = t.n - at < 4 ? (t.n > at ? (int)(t.n - at) : 0) : 4;
        float p[4], g[4], m[4], v[4], root[4];
        get4((const P *)t.p + at, n, wide, p);
        get4((const G *)t.g + at, n, wide, g);
        if constexpr (EIGHT) {
            const unsigned mc = get_codes((const uint8_t *)t.m + at, n, wide), vc = get_codes((const uint8_t *)t.v + at, n, wide);
            decode(mc, t.ms[b], m);
            decode(vc, t.vs[b], v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] * v[i];
        } else {
            get4((const float *)t.m + at, n, wide, m);
            get4((const float *)t.v + at, n, wide, v);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m[i] * a.b1 + g[i] * a.c1;
            v[i] = v[i] * a.b2 + (g[i] * g[i]) * a.c2;
            root[i] = __fsqrt_rn(v[i]);
            p[i] = p[i] * a.keep - __fdiv_rn(m[i], root[i] * a.correction + a.eps) * a.rate;
        }
        put4((P *)t.p + at, n, wide, p);
        if (t.copy) {
            if (t.flags & kCopyF16) put4((f16 *)t.copy + at, n, wide, p);
            else put4((bf16 *)t.copy + at, n, wide, p);
        }
        if constexpr (EIGHT) {
            const float mt = block_max(m), vt = block_max(root);
            // (below 2^-100 the inverse would overflow: such a block is held as zeros)
            const float mi = mt >= 0x1p-100f ? __fdiv_rn(448.0f, mt) : 0.0f, vi = vt >= 0x1p-100f ? __fdiv_rn(448.0f, vt) : 0.0f;
            unsigned mc = 0, vc = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned w = word_of((unsigned long long)t.block0 * kBlock + at + i, a.word0);
                const unsigned c = hold(m[i], mi, w & 0xfffff);
                mc |= (c | (__float_as_uint(m[i]) >> 31) << 7) << (8 * i);
                const unsigned r = hold(root[i], vi, w >> 12);
                vc |= (r == 0 && root[i] > 0.0f ? 1u : r) << (8 * i);
            }
            put_codes((uint8_t *)t.m + at, n, wide, mc);
            put_codes((uint8_t *)t.v + at, n, wide, vc);
            if (lane == 0) {
                t.ms[b] = mt * (float)(1.0 / 448.0);
                t.vs[b] = vt * (float)(1.0 / 448.0);
            }
        } else {
            put4((float *)t.m + at, n, wide, m);
            put4((float *)t.v + at, n, wide, v);
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
    long long total = 0;
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
    a.per_chunk = total > 16 * 4096 ? 16 : total > 4 * 2048 ? 8 : 4;
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
        if (need > 0x7fffffff) return OZIMMU_BAD_ARG;
        if (a.tensors == kTensors || chunks + need > 0x7fffffff || kind[0] != x.param_type || kind[1] != x.grad_type || kind[2] != x.state_type) {
            if (flush() != hipSuccess) return OZIMMU_HIP_ERROR;
            kind[0] = x.param_type;
            kind[1] = x.grad_type;
            kind[2] = x.state_type;
        }
        // four values at a time: 16 bytes of 32 bits, 8 of 16, 4 of 8
        auto off = [](const void *p, int type) { return (uintptr_t)p & (type == OZIMMU_F32 ? 15 : type == OZIMMU_E4M3 ? 3 : 7); };
        const bool wide = !(off(x.param, x.param_type) | off(g, x.grad_type) | off(x.m, x.state_type) | off(x.v, x.state_type) |
                            (x.copy ? off(x.copy, x.copy_type) : 0));
        a.t[a.tensors++] = Tensor{x.param, g, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.count, block0, (int)chunks,
                                  (wide ? kWide : 0) | (x.copy && x.copy_type == OZIMMU_F16 ? kCopyF16 : 0)};
        block0 += blocks;
        chunks += need;
    }
    return flush() == hipSuccess ? OZIMMU_OK : OZIMMU_HIP_ERROR;
}

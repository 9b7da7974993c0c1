// The tiled matrix product of the feed-forward operators: D[q][p] = act(sum_k P Q + bias) + residual.
//
// A work-group owns a tile of BP x BQ entries and walks k in steps of 128 bytes of an operand's row (64 entries of 16
// bits, 32 of 32 bits).  Both operands of a step stand in LDS as BP (BQ) * 128 bytes, two stages of them: the copies of
// step t + 1 are issued behind the barrier that opens step t and have all of its products to arrive, one barrier a step.
//
// k_rows: the entries of an operand's row are contiguous along k (activations and weights of a forward pass).  LDS row r
//   holds its 8 chunks of 16 bytes at position chunk ^ (r / 2 % 8): the 16 rows that a matrix instruction's operand takes
//   then lie in 16 different chunks of 256 bytes, so that a 16-byte read meets no bank twice.
// otherwise: k is the slow index of the operand in memory (weights in dx, both operands in dw).  LDS keeps that order, a
//   row per k, and for 16 bits the read itself transposes (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 entries, lane i
//   gets entry i of each); 32-byte units are placed at unit ^ (k % 4 + 4 (k / 8 % 2)), the eight rows that half a
//   wavefront reads in eight different units of 256 bytes.  For 32 bits a lane reads single entries, 64-byte units
//   at unit ^ (k / 4 % 4).
//
// DIRECT: the copies go from memory to LDS without registers, which wants 16-byte alignment of every row; what lies
// behind k is read from a chunk of zeros.  Otherwise 16 bytes a lane are loaded at any alignment, and written to LDS behind the
// products.  Rows behind the operand's last are read as the last and not stored.
#pragma once
#include "few_dev.h"

namespace oz {

__device__ __attribute__((aligned(16))) const unsigned kZeroChunk[4] = {0, 0, 0, 0};

// 16 bytes per lane, any global address -> LDS (ldsaddr + lane * 16)
__device__ __forceinline__ void lds_dma16_any(const void *p, unsigned ldsaddr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(ldsaddr), "v"(p) : "memory", "m0");
}

template <class T, int BP, int BQ, int WP, int WQ>
struct ProductShape {
    static constexpr int kWaves = WP * WQ, kThreads = 64 * kWaves;
    static constexpr int kStage = (BP + BQ) * 128;
    static constexpr int kPW = BP / WP, kQW = BQ / WQ;                  // a wavefront's part of the tile
    static constexpr int kStripLd = kPW + 4;                            // floats; epilogue strip of 16 q a wavefront
    static constexpr int kStrip = kWaves * 16 * kStripLd * 4;
    static constexpr int kLds = 2 * kStage > kStrip ? 2 * kStage : kStrip;
};

// One operand of the tile: where its chunks come from and where they go in LDS.
template <class T, bool K_ROWS, int B, int WAVES, bool DIRECT>
struct Operand {
    static constexpr int E = Chunk<T>::E, KE = 8 * E;                   // entries of a chunk, of a step
    static constexpr int N = B * 8 / (64 * WAVES);                      // chunks a lane copies per step
    static constexpr int kRowBytes = K_ROWS ? 128 : B * (int)sizeof(T); // of an LDS row
    static constexpr int kRowChunks = kRowBytes / 16;
    static_assert(N * 64 * WAVES == B * 8, "whole chunks");

    const T *base;
    int ld, rows, row0, nk;
    unsigned off[DIRECT ? N : 1];                                       // bytes behind the step's base
    v4u reg[DIRECT ? 1 : N];

    static __device__ __forceinline__ int place(int c)                  // LDS row's chunk -> chunk of the row in memory
    {
        return c;
    }
    // swizzle of 16-byte chunks in LDS row r
    static __device__ __forceinline__ int twist(int r)
    {
        if constexpr (K_ROWS) return (r >> 1) & 7;
        else if constexpr (sizeof(T) == 2) return (((r & 3) | ((r >> 1) & 4)) << 1) & (kRowChunks - 1);
        else return (((r >> 2) & 3) << 2) & (kRowChunks - 1);
    }
    static __device__ __forceinline__ void slot(int i, int wave, int lane, int &r, int &c)
    {
        const int s = (i * WAVES + wave) * 64 + lane;                   // chunk in LDS order
        r = s / kRowChunks;
        c = (s % kRowChunks) ^ twist(r);
    }

    __device__ __forceinline__ void init(const void *p, int ld_, int rows_, int row0_, int nk_, int wave, int lane)
    {
        base = (const T *)p;
        ld = ld_;
        rows = rows_;
        row0 = row0_;
        nk = nk_;
        if constexpr (DIRECT) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int r, c;
                slot(i, wave, lane, r, c);
                if constexpr (K_ROWS) {
                    const int row = row0 + r < rows ? r : rows - 1 - row0;
                    off[i] = (unsigned)row * (unsigned)ld * (unsigned)sizeof(T) + c * 16;
                } else {
                    const int col = row0 + c * E < rows ? c * E : rows - E - row0;   // (rows is a multiple of E)
                    off[i] = (unsigned)r * (unsigned)ld * (unsigned)sizeof(T) + col * (int)sizeof(T);
                }
            }
        }
    }

    __device__ __forceinline__ const T *at(int k0) const
    {
        return K_ROWS ? base + (size_t)row0 * ld + k0 : base + (size_t)k0 * ld + row0;
    }

    // DIRECT: issue the copies of the step that starts at k0
    __device__ __forceinline__ void copy(int k0, unsigned lds, int wave, int lane)
    {
        const T *p = at(k0);
        if (k0 + KE <= nk) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds_dma16(p, off[i], lds + (i * WAVES + wave) * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int r, c;
                slot(i, wave, lane, r, c);
                const bool in = (K_ROWS ? k0 + c * E : k0 + r) < nk;
                lds_dma16_any(in ? (const void *)((const char *)p + off[i]) : (const void *)kZeroChunk, lds + (i * WAVES + wave) * 1024);
            }
        }
    }

    __device__ __forceinline__ void load(int k0, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int r, c;
            slot(i, wave, lane, r, c);
            if constexpr (K_ROWS) {
                const int row = row0 + r < rows ? row0 + r : rows - 1, k = k0 + c * E;
                reg[i] = load_chunk(base + (size_t)row * ld + k, nk - k);
            } else {
                const int k = k0 + r, col = row0 + c * E;
                reg[i] = load_chunk(base + (size_t)k * ld + col, k < nk ? rows - col : 0);
            }
        }
    }
    __device__ __forceinline__ void store(char *lds, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) *(v4u *)(lds + ((i * WAVES + wave) * 64 + lane) * 16) = reg[i];
    }

    // the operand of rows w0 + 16 f ... + 15 (w0: a wavefront's part, a multiple of 32), half s of the step
    static __device__ __forceinline__ v4u fragment(const char *lds, int w0, int f, int s, int lane)
    {
        const int r = lane & 15, g = lane >> 4;
        if constexpr (K_ROWS) {
            const int row = w0 + 16 * f + r;
            return *(const v4u *)(lds + row * 128 + ((((4 * s + g) ^ ((r >> 1) & 7))) << 4));
        } else if constexpr (sizeof(T) == 2) {
            typedef short v4s __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4s lds_v4s;
            const int k = 32 * s + 8 * g + (r >> 2);
            const int unit = ((w0 >> 4) + f) ^ (twist(k) >> 1);
            const char *p = lds + k * kRowBytes + unit * 32 + (r & 3) * 8;
            union { v4s h[2]; v4u v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(p + 4 * kRowBytes));
            return u.v;
        } else {
            const int col = w0 + 16 * f + r;
            v4u v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 16 * s + 4 * g + i;
                v[i] = *(const unsigned *)(lds + k * kRowBytes + (((col >> 2) ^ twist(k)) << 4) + (col & 3) * 4);
            }
            return v;
        }
    }
};

template <class T, bool PK, bool QK, int BP, int BQ, int WP, int WQ, bool DIRECT>
__global__ __launch_bounds__(64 * WP * WQ) void product_kernel(Product a, float *partial, int steps_per_split, int tiles_p, int tiles_q)
{
    using S = ProductShape<T, BP, BQ, WP, WQ>;
    constexpr int FP = S::kPW / 16, FQ = S::kQW / 16, KE = 8 * Chunk<T>::E;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    int tq, tp;
    if (!tile_of_block_xcd(blockIdx.x, tiles_q, tiles_p, false, tq, tp)) return;
    const int wp = wave % WP * S::kPW, wq = wave / WP * S::kQW;

    Operand<T, PK, BP, S::kWaves, DIRECT> P;
    Operand<T, QK, BQ, S::kWaves, DIRECT> Q;
    P.init(a.P, a.ldp, a.e.np, tp * BP, a.nk, wave, lane);
    Q.init(a.Q, a.ldq, a.e.nq, tq * BQ, a.nk, wave, lane);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    v4f acc[FP][FQ];
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
        for (int j = 0; j < FQ; ++j) acc[i][j] = v4f{0, 0, 0, 0};

    const int all = (a.nk + KE - 1) / KE;
    const int t0 = (int)blockIdx.y * steps_per_split, t1 = all < t0 + steps_per_split ? all : t0 + steps_per_split;

    auto products = [&](const char *stage) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            v4u p[FP], q[FQ];
#pragma unroll
            for (int j = 0; j < FQ; ++j) q[j] = Q.fragment(stage + BP * 128, wq, j, s, lane);
#pragma unroll
            for (int i = 0; i < FP; ++i) p[i] = P.fragment(stage, wp, i, s, lane);
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j) acc[i][j] = mma(p[i], q[j], acc[i][j], T{});
        }
    };

    if (t0 < t1) {
        if constexpr (DIRECT) {
            P.copy(t0 * KE, lds0, wave, lane);
            Q.copy(t0 * KE, lds0 + BP * 128, wave, lane);
            for (int t = t0; t < t1; ++t) {
                const int now = (t - t0) & 1;
                wait_vmcnt<0>();
                __syncthreads();                    // the step's copies are there, and nobody reads the other stage any more
                if (t + 1 < t1) {
                    const unsigned to = lds0 + (now ^ 1) * S::kStage;
                    P.copy((t + 1) * KE, to, wave, lane);
                    Q.copy((t + 1) * KE, to + BP * 128, wave, lane);
                }
                products(lds + now * S::kStage);
            }
        } else {
            P.load(t0 * KE, wave, lane);
            Q.load(t0 * KE, wave, lane);
            P.store(lds, wave, lane);
            Q.store(lds + BP * 128, wave, lane);
            for (int t = t0; t < t1; ++t) {
                const int now = (t - t0) & 1;
                __syncthreads();
                if (t + 1 < t1) {
                    P.load((t + 1) * KE, wave, lane);
                    Q.load((t + 1) * KE, wave, lane);
                }
                products(lds + now * S::kStage);
                if (t + 1 < t1) {
                    char *to = lds + (now ^ 1) * S::kStage;
                    P.store(to, wave, lane);
                    Q.store(to + BP * 128, wave, lane);
                }
            }
        }
    }

    // Epilogue: 16 q of a wavefront's part at a time pass through LDS, so that a lane has 8 entries along p.
    __syncthreads();
    float *strip = (float *)lds + wave * 16 * S::kStripLd;
    const int r = lane & 15, g = lane >> 4;
    constexpr int kRowLanes = S::kPW / 8, kRows = 64 / kRowLanes;
    static_assert(16 % kRows == 0, "");
    for (int jj = 0; jj < FQ; ++jj) {
        static_for<0, FQ>([&](auto J) {
            if (J == jj)
#pragma unroll
                for (int i = 0; i < FP; ++i) *(v4f *)(strip + r * S::kStripLd + 16 * i + 4 * g) = acc[i][J];
        });
        __builtin_amdgcn_wave_barrier();
#pragma nounroll
        for (int y = 0; y < 16; y += kRows) {
            const int row = y + lane / kRowLanes, col = lane % kRowLanes * 8;
            const int q = tq * BQ + wq + 16 * jj + row, p = tp * BP + wp + col;
            float v[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v4f x = *(const v4f *)(strip + row * S::kStripLd + col + 4 * i);
#pragma unroll
                for (int c = 0; c < 4; ++c) v[4 * i + c] = x[c];
            }
            if (q >= a.e.nq || p >= a.e.np) continue;
            if (partial) {
                // (partial sums: rows of np rounded up to 8 floats, so that they are written whole)
                const int ldn = (a.e.np + 7) & ~7;
                float *to = partial + ((size_t)blockIdx.y * a.e.nq + q) * ldn + p;
                *(v4f *)to = v4f{v[0], v[1], v[2], v[3]};
                *(v4f *)(to + 4) = v4f{v[4], v[5], v[6], v[7]};
            } else {
                finish_row<T>(a.e, q, p, v);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// the sums of the parts, in their order, and the epilogue
template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(Epilogue e, const float *partial, int splits)
{
    const int groups = (e.np + 7) / 8;
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (size_t)groups * e.nq) return;
    const int q = (int)(at / groups), p = (int)(at % groups) * 8;
    const size_t plane = (size_t)e.nq * groups * 8;
    const float *from = partial + (size_t)q * groups * 8 + p;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int s = 0; s < splits; ++s) {
        const v4f a = *(const v4f *)(from + s * plane), b = *(const v4f *)(from + s * plane + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] += a[i];
            v[4 + i] += b[i];
        }
    }
    finish_row<T>(e, q, p, v);
}

template <class T, bool PK, bool QK, int BP, int BQ, int WP, int WQ, bool DIRECT>
hipError_t launch_product_shape(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    using S = ProductShape<T, BP, BQ, WP, WQ>;
    const int tiles_p = (a.e.np + BP - 1) / BP, tiles_q = (a.e.nq + BQ - 1) / BQ;
    const long long blocks = tile_order_blocks(tiles_q, tiles_p, false);
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const auto kernel = product_kernel<T, PK, QK, BP, BQ, WP, WQ, DIRECT>;
    static std::atomic<unsigned long long> done{0};
    if (hipError_t e = allow_dynamic_lds((const void *)kernel, S::kLds, done)) return e;
    kernel<<<dim3((unsigned)blocks, plan.splits), S::kThreads, S::kLds, st>>>(a, plan.splits > 1 ? partial : nullptr, plan.steps, tiles_p, tiles_q);
    return hipGetLastError();
}

template <class T, bool PK, bool QK>
hipError_t launch_product_order(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    if (plan.direct) {
        if constexpr (sizeof(T) == 2)
            if (plan.tile == 0) return launch_product_shape<T, PK, QK, 256, 256, 2, 4, true>(a, plan, partial, st);
        if (plan.tile == 1) return launch_product_shape<T, PK, QK, 128, 128, 2, 2, true>(a, plan, partial, st);
        return launch_product_shape<T, PK, QK, 64, 64, 2, 2, true>(a, plan, partial, st);
    }
    if (plan.tile <= 1) return launch_product_shape<T, PK, QK, 128, 128, 2, 2, false>(a, plan, partial, st);
    return launch_product_shape<T, PK, QK, 64, 64, 2, 2, false>(a, plan, partial, st);
}

template <class T>
hipError_t launch_product_tiles(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    if (a.p_k_rows && a.q_k_rows) return launch_product_order<T, true, true>(a, plan, partial, st);
    if (a.q_k_rows) return launch_product_order<T, false, true>(a, plan, partial, st);
    return launch_product_order<T, false, false>(a, plan, partial, st);
}

template <class T>
hipError_t launch_join(const Product &a, const ProductPlan &plan, const float *partial, hipStream_t st)
{
    const size_t threads = (size_t)a.e.nq * ((a.e.np + 7) / 8), groups = (threads + 255) / 256;
    if (groups > 0x7fffffff) return hipErrorInvalidValue;
    product_join_kernel<T><<<(unsigned)groups, 256, 0, st>>>(a.e, partial, plan.splits);
    return hipGetLastError();
}

template <class T>
hipError_t launch_product_type(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    if (hipError_t e = plan.tile == kTileFew ? launch_few_tokens<T>(a, plan, partial, st) : launch_product_tiles<T>(a, plan, partial, st)) return e;
    return plan.splits > 1 ? launch_join<T>(a, plan, partial, st) : hipSuccess;
}

}  // namespace oz

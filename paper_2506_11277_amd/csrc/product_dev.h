// The tiled matrix product of the feed-forward operators: D[q][p] = act(sum_k P Q + bias) + residual.
//
// A work-group owns a tile of BP x BQ entries and walks k in steps of 128 bytes of an operand's row (128 entries of 8 bits, 64 of 16
// bits, 32 of 32 bits).  Both operands of a step stand in LDS as BP (BQ) * 128 bytes, in a ring of two stages (256 x 256: all
// that fits) or four: the copies of a step are issued one to three steps before its products, one barrier a step.  (Gradients in 32 bits also take 32 x 64.)
//
// What bounds it: 256 x 256 in 16 bits the matrix instructions at the clock that the board's power leaves them, with LDS (128 KB read
// and 64 written a step of 2048 cycles of matrix instructions) close behind: 8192^3 bf16 1.43 PFLOP/s, 4096^3 1.36, 8192 x 4096 x 8192
// with a gelu and `pre` 1.2.  128 x 128 and 64 x 64 LDS: 96 and 48 KB a step of 512 and 128 cycles (2048^3 770 TFLOP/s,
// 1024^3 260).  32 bits: the matrix instructions (2048^3 133 TFLOP/s, 4096^3 140).
//
// 8 bits, results in 16: a step takes as long as in 16 bits, with twice the k.  8192 x 4096 x 8192 211 us (2.6 POP/s; without an epilogue 195),
// with gelu and `pre` 239 to 252 from card to card, 16384 of k 2.9 POP/s; on operands of zeros a step takes a quarter less: power.  A tile's epilogue is 5 us of
// vector instructions (10 with gelu), and as long goes by until its first products: four times in 8192 x 8192.
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
// products: twice the time of a step, so larger operands are copied to aligned rows first (pad.hip).  Rows behind the
// operand's last are read as the last and not stored.
#pragma once
#include "few_dev.h"

namespace oz {

__device__ __attribute__((aligned(16))) const unsigned kZeroChunk[4] = {0, 0, 0, 0};

// 16 bytes per lane, any global address -> LDS (ldsaddr + lane * 16)
__device__ __forceinline__ void lds_dma16_any(const void *p, unsigned ldsaddr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(ldsaddr), "v"(p) : "memory", "m0");
}

// c[j] += p q[j] as mma(), in place and where the order in the source puts it.  (The builtin lets the register allocator move
// accumulators about: 184 moves in a step of 128 instructions and 758 us instead of 490 for 8192 x 4096 x 8192 with 256 x 256
// tiles, 110 moves in a step of 32 with 128 x 128.)  ACC: c in accumulator registers, else in ordinary ones; the
// largest tile takes both, so that the allocator has some of either to spare.  settle() has to follow before anything else
// reads c, and the same c is not used again within the next instruction.
template <bool ACC>
__device__ __forceinline__ void mma_one(v4u p, v4u q, v4f &c, bf16)
{
    if constexpr (ACC) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
    else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(p), "v"(q));
}
template <bool ACC>
__device__ __forceinline__ void mma_one(v4u p, v4u q, v4f &c, f16)
{
    if constexpr (ACC) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
    else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(c) : "v"(p), "v"(q));
}
template <bool ACC>
__device__ __forceinline__ void mma_one(v4u p, v4u q, v4f &c, int8_t)
{
    if constexpr (ACC) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
    else asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+v"(c) : "v"(p), "v"(q));
}
template <bool ACC, class T, int FQ>
__device__ __forceinline__ void mma_row(v4u p, const v4u (&q)[FQ], v4f (&c)[FQ])
{
    static_assert(FQ >= 2, "");
    if constexpr (sizeof(T) <= 2) {
#pragma unroll
        for (int j = 0; j < FQ; ++j) mma_one<ACC>(p, q[j], c[j], T{});
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < FQ; ++j) asm volatile("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+v"(c[j]) : "v"(p[e]), "v"(q[j][e]));
    }
}
// the wait states between a matrix instruction and another use of its result, which the compiler does not see through the asm: once, behind
// the last of them (WAIT), and for what came before it the place alone
template <bool ACC, bool WAIT, int N>
__device__ __forceinline__ void settle(v4f (&c)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 2) {
        if (WAIT && j == 0) asm volatile("s_nop 15\n\ts_nop 15");
        if constexpr (ACC) asm volatile("" : "+a"(c[j]), "+a"(c[j + 1]));
        else asm volatile("" : "+v"(c[j]), "+v"(c[j + 1]));
    }
}

template <class T, int BP, int BQ, int WP, int WQ>
struct ProductShape {
    static constexpr int kWaves = WP * WQ, kThreads = 64 * kWaves;
    static constexpr int kStage = (BP + BQ) * 128;
    static constexpr int kPW = BP / WP, kQW = BQ / WQ;                  // a wavefront's part of the tile
    static constexpr bool kAlone = kPW == 128 && kQW == 128;            // one wavefront per SIMD
    static constexpr int kSQ = kQW < 64 ? kQW : 64;                     // epilogue: q of a wavefront's part at a time
    static constexpr int kSumsLd = kPW + 4, kSums = kSQ * kSumsLd * 4;
    static constexpr int kStages = kAlone ? 2 : 4;
    // behind stages and sums, for operands of 8 bits: the scales of Q's rows
    static constexpr int kRows = kStages * kStage > kWaves * kSums ? kStages * kStage : kWaves * kSums;
    static constexpr int kLds = kRows + (sizeof(T) == 1 ? BQ * 4 : 0);
    static_assert(kLds <= kLdsBytes, "LDS");
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
    v4u reg[2][DIRECT ? 1 : N];                                         // chunks on their way to LDS, of two steps

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

    // one of the N copies of a step that lies before nk; from = at(its k)
    template <int I>
    __device__ __forceinline__ void copy_one(const T *from, unsigned lds, int wave)
    {
        lds_dma16(from, off[I], lds + (I * WAVES + wave) * 1024);
    }

    template <int S>
    __device__ __forceinline__ void load(int k0, int wave, int lane)
    {
        if (k0 + KE <= nk && (K_ROWS || row0 + B <= rows)) {            // (the same for all lanes)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int r, c;
                slot(i, wave, lane, r, c);
                const T *from = K_ROWS ? base + (size_t)(row0 + r < rows ? row0 + r : rows - 1) * ld + k0 + c * E : base + (size_t)(k0 + r) * ld + row0 + c * E;
                __builtin_memcpy(&reg[S][i], from, 16);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int r, c;
            slot(i, wave, lane, r, c);
            if constexpr (K_ROWS) {
                const int row = row0 + r < rows ? row0 + r : rows - 1, k = k0 + c * E;
                reg[S][i] = load_chunk(base + (size_t)row * ld + k, nk - k, k);
            } else {
                const int k = k0 + r, col = row0 + c * E;
                reg[S][i] = load_chunk(base + (size_t)k * ld + col, k < nk ? rows - col : 0);
            }
        }
    }
    template <int S>
    __device__ __forceinline__ void store(char *lds, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) *(v4u *)(lds + ((i * WAVES + wave) * 64 + lane) * 16) = reg[S][i];
    }

    // Where a lane finds its operands in a stage: fragment() of rows w0 + 16 f ... + 15 (w0: a wavefront's part, a multiple of
    // 16) and half h of a step is read from `from`, which is reader() behind the operand's place in LDS (a multiple of 1 KB); f
    // and the swizzle meet in one exclusive or.
    static __device__ __forceinline__ unsigned reader(int w0, int lane)
    {
        const int r = lane & 15, g = lane >> 4;
        if constexpr (K_ROWS) return (w0 + r) * 128 + ((g ^ twist(r)) << 4);
        else if constexpr (sizeof(T) == 2) {
            const int k = 8 * g + (r >> 2);
            return k * kRowBytes + (((w0 >> 4) ^ (twist(k) >> 1)) << 5) + (r & 3) * 8;
        } else return 4 * g * kRowBytes + ((((w0 + r) >> 2) ^ twist(4 * g)) << 4) + (r & 3) * 4;
    }
    static __device__ __forceinline__ v4u fragment(unsigned from, int f, int h)
    {
        if constexpr (K_ROWS) {
            return *(const __attribute__((address_space(3))) v4u *)((from ^ (h << 6)) + f * 2048);
        } else if constexpr (sizeof(T) == 2) {
            typedef short v4s __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4s lds_v4s;
            const unsigned at = (from ^ (f << 5)) + h * 32 * kRowBytes;
            const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)at), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(at + 4 * kRowBytes));
            const v2u a = __builtin_bit_cast(v2u, x), b = __builtin_bit_cast(v2u, y);
            return v4u{a[0], a[1], b[0], b[1]};
        } else {
            const unsigned at = (from ^ (f << 6)) + h * 16 * kRowBytes;
            v4u v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *(const __attribute__((address_space(3))) unsigned *)(at + i * kRowBytes);
            return v;
        }
    }
};

// Epilogue of a wavefront's part of the tile: its sums pass through LDS, 64 q of it at a time (a loop over them with the
// accumulators in registers would have to pick them by number, which puts them in memory), so that a lane has 8
// entries along p of a row, always of the same columns: its bias is loaded once.
template <class T>
struct Columns {
    float bias[8], scale[sizeof(T) == 1 ? 8 : 1];
};
template <class T, class Out, int PW>
__device__ __forceinline__ void load_columns(const Epilogue &e, int p0, int lane, Columns<T> &c)
{
    const int p = p0 + lane % (PW / 8) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) c.bias[i] = 0.0f;
    if (sizeof(T) > 1 && e.bias && e.wide && p + 8 <= e.np) load_row((const Out *)e.bias + p, c.bias);
    if constexpr (sizeof(T) == 1) {
        RowVectors<Out> with;
        with.load_columns(e, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c.bias[i] = with.bias[i];
            c.scale[i] = with.scale[i];
        }
    }
}

// rows q0 ... q0 + QW - 1 of `sums`, PW + 4 floats apart; R rows of a lane at a time.  QS: rows may have a scale.
// !WHOLE: rows at any alignment, what lies behind their last entry one by one (8-bit operands; entry by entry 1531 x 1001 -> 777 takes 18.8 us instead
// of 14.3, 4097 x 1001 -> 4095 84 instead of 57, but what is aligned would take 221 instead of 210 this way, 8192 x 4096 -> 8192)
template <class T, class Out, bool QS, int ACT, int PW, int QW, bool WHOLE = true>
__device__ __forceinline__ void epilogue_rows(const Epilogue &e, float *partial, const Columns<T> &columns, const float *sums, const float *rows, int q0, int p0, int lane)
{
    constexpr int LD = PW + 4, LANES = PW / 8, ROWS = 64 / LANES, MOST = sizeof(T) == 1 ? 8 : 4, R = QW / ROWS < MOST ? QW / ROWS : MOST;
    static_assert(QW % (ROWS * R) == 0, "");
    const int col = lane % LANES * 8, p = p0 + col;
    if (p >= e.np) return;
    auto write = [&](Out *to, const float (&x)[8]) __attribute__((always_inline)) {
        if constexpr (!WHOLE) store8(to, e.np - p, x);
        else if constexpr (PW == 128) stream_row(to, x);
        else store_row(to, x);
    };
#pragma nounroll
    for (int s = lane / LANES; s < QW && q0 + s < e.nq; s += R * ROWS) {
        float v[R][8], res[R][8];
#pragma unroll
        for (int y = 0; y < R; ++y)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[y][i] = sums[(s + y * ROWS) * LD + col + i];
        if (partial) {
            // (partial sums: rows of np rounded up to 8 floats, so that they are written whole)
            const int ldn = (e.np + 7) & ~7;
#pragma unroll
            for (int y = 0; y < R; ++y)
                if (q0 + s + y * ROWS < e.nq) store_row(partial + ((size_t)blockIdx.y * e.nq + q0 + s + y * ROWS) * ldn + p, v[y]);
            continue;
        }
        float x[R];
#pragma unroll
        for (int y = 0; y < R; ++y) {
            x[y] = 1.0f;
            if (sizeof(T) == 1) x[y] = rows[s + y * ROWS];
            else if (QS && e.q_scale && q0 + s + y * ROWS < e.nq) x[y] = e.q_scale[q0 + s + y * ROWS];
        }
        if (e.residual)
#pragma unroll
            for (int y = 0; y < R; ++y)
                if (q0 + s + y * ROWS < e.nq) {
                    const Out *from = (const Out *)e.residual + (size_t)(q0 + s + y * ROWS) * e.ldr + p;
                    if constexpr (WHOLE) {
                        load_row(from, res[y]);
                    } else {
                        Eight<Out> t;
                        t.load(from, e.np - p);
#pragma unroll
                        for (int i = 0; i < 8; ++i) res[y][i] = t[i];
                    }
                }
#pragma unroll
        for (int y = 0; y < R; ++y) {
            const int q = q0 + s + y * ROWS;
            if (q >= e.nq) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[y][i] = scaled<T>(v[y][i], x[y], columns.scale[sizeof(T) == 1 ? i : 0], columns.bias[i]);
            if (e.pre) write((Out *)e.pre + (size_t)q * e.ldpre + p, v[y]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[y][i] = activate_sum<T, Out>(ACT, v[y][i]);
            if (e.residual)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[y][i] += res[y][i];
            write((Out *)e.out + (size_t)q * e.ldo + p, v[y]);
        }
    }
}

// ... entry by entry, where rows are not aligned or end within 8 entries (operands of 16 and 32 bits): consecutive lanes take consecutive entries, four
// rows at a time; all 16 of a lane in a 64 x 64 tile (1531 x 1008 x 777 f16 with a residual 11.8 us against 12.2; in a 128 x 128
// tile more than four are slower, 4097 x 1024 x 4095 f16 166 us against 155)
template <class T, class Out, bool QS, int ACT, int PW, int QW>
__device__ __forceinline__ void epilogue_entries(const Epilogue &e, const float *sums, int q0, int p0, int lane)
{
    constexpr int LD = PW + 4, W = PW < 64 ? PW : 64, ROWS = 64 / W, R = PW == 32 ? 16 : 4;
    static_assert(sizeof(T) > 1 && QW % (ROWS * R) == 0, "");
#pragma nounroll
    for (int c = lane % W; c < PW; c += W) {
        const int p = p0 + c;
        if (p >= e.np) break;
        const float bias = e.bias ? (float)((const Out *)e.bias)[p] : 0.0f;
#pragma nounroll
        for (int s = lane / W; s < QW && q0 + s < e.nq; s += R * ROWS) {
            float v[R], res[R];
#pragma unroll
            for (int y = 0; y < R; ++y) {
                const int q = q0 + s + y * ROWS;
                v[y] = scaled<T>(sums[(s + y * ROWS) * LD + c], QS && e.q_scale && q < e.nq ? e.q_scale[q] : 1.0f, 1.0f, bias);
                res[y] = e.residual && q < e.nq ? (float)((const Out *)e.residual)[(size_t)q * e.ldr + p] : 0.0f;
            }
#pragma unroll
            for (int y = 0; y < R; ++y) {
                const int q = q0 + s + y * ROWS;
                if (q >= e.nq) continue;
                if (e.pre) ((Out *)e.pre)[(size_t)q * e.ldpre + p] = (Out)v[y];
                float x = activate<Out>(ACT, v[y]);
                if (e.residual) x += res[y];
                ((Out *)e.out)[(size_t)q * e.ldo + p] = (Out)x;
            }
        }
    }
}

template <class T, class Out, bool QS, int ACT, int PW, int QW>
__device__ __forceinline__ void epilogue_as(const Epilogue &e, float *partial, const Columns<T> &columns, const float *sums, const float *rows, int q0, int p0, int lane)
{
    if (partial || (e.wide && (p0 + PW <= e.np || e.np % 8 == 0))) epilogue_rows<T, Out, QS, ACT, PW, QW>(e, partial, columns, sums, rows, q0, p0, lane);
    else if constexpr (sizeof(T) == 1) epilogue_rows<T, Out, QS, ACT, PW, QW, false>(e, partial, columns, sums, rows, q0, p0, lane);
    else epilogue_entries<T, Out, QS, ACT, PW, QW>(e, sums, q0, p0, lane);
}

template <class T, class Out, bool QS, int PW, int QW>
__device__ __forceinline__ void epilogue(const Epilogue &e, float *partial, const Columns<T> &columns, const float *sums, const float *rows, int q0, int p0, int lane)
{
    switch (e.act) {                                // (decided once: a lane's entries decide nothing)
        case OZIMMU_ACT_RELU: return epilogue_as<T, Out, QS, OZIMMU_ACT_RELU, PW, QW>(e, partial, columns, sums, rows, q0, p0, lane);
        case OZIMMU_ACT_GELU: return epilogue_as<T, Out, QS, OZIMMU_ACT_GELU, PW, QW>(e, partial, columns, sums, rows, q0, p0, lane);
        case OZIMMU_ACT_GELU_TANH: return epilogue_as<T, Out, QS, OZIMMU_ACT_GELU_TANH, PW, QW>(e, partial, columns, sums, rows, q0, p0, lane);
        case OZIMMU_ACT_SILU: return epilogue_as<T, Out, QS, OZIMMU_ACT_SILU, PW, QW>(e, partial, columns, sums, rows, q0, p0, lane);
    }
    epilogue_as<T, Out, QS, OZIMMU_ACT_NONE, PW, QW>(e, partial, columns, sums, rows, q0, p0, lane);
}

// one tile, or one part of its contraction
template <class T, class Out, bool PK, bool QK, int BP, int BQ, int WP, int WQ, bool DIRECT>
__device__ __forceinline__ void product_tile(const Product &a, float *partial, int steps_per_split, int tiles_p, int tiles_q, int block, char *lds)
{
    using S = ProductShape<T, BP, BQ, WP, WQ>;
    constexpr int FP = S::kPW / 16, FQ = S::kQW / 16, KE = 8 * Chunk<T>::E;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wp = wave % WP * S::kPW, wq = wave / WP * S::kQW;
    int tq, tp;
    if (!tile_of_block_xcd(block, tiles_q, tiles_p, false, tq, tp)) return;

    Operand<T, PK, BP, S::kWaves, DIRECT> P;
    Operand<T, QK, BQ, S::kWaves, DIRECT> Q;
    P.init(a.P, a.ldp, a.p_rows, tp * BP, a.p_nk, wave, lane);
    Q.init(a.Q, a.ldq, a.q_rows, tq * BQ, a.q_nk, wave, lane);
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;

    // (a load in the epilogue waits for all stores before it)
    if constexpr (sizeof(T) == 1) {
        static_assert(BQ <= S::kThreads, "a row a thread");
        const int t = threadIdx.x;
        if (t < BQ) ((float *)(lds + S::kRows))[t] = tq * BQ + t < a.e.nq ? a.e.q_scale[tq * BQ + t] : 0.0f;
    }

    v4f acc[FP][FQ];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FQ; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    };

    const int all = (a.nk + KE - 1) / KE;
    const int t0 = (int)blockIdx.y * steps_per_split, t1 = all < t0 + steps_per_split ? all : t0 + steps_per_split;

    v4u p[2][FP], q[2][FQ];                         // operands of the two halves of a step
    const unsigned pbase = lds0 + P.reader(wp, lane), qbase = lds0 + BP * 128 + Q.reader(wq, lane);
    // (hidden from the optimiser, which otherwise keeps every fragment's address in a register of its own)
    auto in_stage = [&](unsigned base, int stage) __attribute__((always_inline)) {
        unsigned from = base + stage * S::kStage;
        asm volatile("" : "+v"(from));
        return from;
    };
    auto read = [&](int stage, auto H) __attribute__((always_inline)) {
        const unsigned fp = in_stage(pbase, stage), fq = in_stage(qbase, stage);
#pragma unroll
        for (int j = 0; j < FQ; ++j) q[H][j] = Q.fragment(fq, j, H);
#pragma unroll
        for (int i = 0; i < FP; ++i) p[H][i] = P.fragment(fp, i, H);
    };
    auto products = [&](auto H) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FQ; ++j) acc[i][j] = mma(p[H][i], q[H][j], acc[i][j], T{});
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};

    auto copy = [&](int t, int stage) __attribute__((always_inline)) {
        P.copy(t * KE, lds0 + stage * S::kStage, wave, lane);
        Q.copy(t * KE, lds0 + stage * S::kStage + BP * 128, wave, lane);
    };

    clear();
    if constexpr (DIRECT) {
        // With one to two wavefronts per SIMD little but a wavefront's own matrix instructions hides its reads, so every read and
        // copy has its place among them.  While the products of a half step run, the operands of the other half are read,
        // three reads to a row of instructions; behind the barrier in the middle of a step its second half's operands are in
        // registers, so the copies of the step kStages on take its stage, two to a row (more at once wait for each other in the
        // address unit, and the wavefront with them: 472 us instead of 437 with 256 x 256 tiles).
        constexpr int R = S::kStages, L = P.N + Q.N;                    // L: copies of a step
        constexpr std::integral_constant<bool, true> reads{};
        constexpr std::integral_constant<bool, false> none{};
        auto half = [&](auto H, auto READ, int stage, auto &&copies) __attribute__((always_inline)) {
            constexpr int O = 1 - H;
            const unsigned fp = in_stage(pbase, stage), fq = in_stage(qbase, stage);
            static_for<0, FP>([&](auto I) __attribute__((always_inline)) {
                if constexpr (READ)
                    static_for<3 * I, 3 * I + 3>([&](auto X) __attribute__((always_inline)) {
                        if constexpr (X < FQ) q[O][X] = Q.fragment(fq, X, O);
                        else if constexpr (X < FQ + FP) p[O][X - FQ] = P.fragment(fp, X - FQ, O);
                    });
                copies(I);
                __builtin_amdgcn_sched_barrier(0);
                mma_row<(S::kAlone && I < FP - 1), T>(p[H][I], q[H], acc[I]);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        constexpr int A = (L + FP - 1) / FP;        // copies to a row: two, of 32 x 64 three
        static_assert(3 * FP >= FP + FQ && A <= 3, "reads and copies of a step");
        auto nothing = [](auto) __attribute__((always_inline)) {};
        // (every part of the contraction has a step)
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (t0 + i < t1) copy(t0 + i, i);
        if (t0 + R <= t1) wait_vmcnt<(R - 1) * L>();
        else wait_vmcnt<0>();
        __syncthreads();
        read(0, first);
        int t = t0, now = 0;
        // (steps whose R-th next is there and whole)
        const int whole = a.nk / KE < t1 ? a.nk / KE : t1;
        for (int left = whole - R - t0; left > 0; --left, ++t) {
            const int next = now + 1 == R ? 0 : now + 1;
            half(first, reads, now, nothing);
            // the next step's copies are there, and nobody reads this step's stage any more
            wait_vmcnt<(R - 2) * L>();
            __syncthreads();
            const T *from_p = P.at((t + R) * KE), *from_q = Q.at((t + R) * KE);
            const unsigned to = lds0 + now * S::kStage;
            half(second, reads, next, [&](auto I) __attribute__((always_inline)) {
                static_for<A * I, A * I + A>([&](auto C) __attribute__((always_inline)) {
                    if constexpr (C < P.N) P.template copy_one<C>(from_p, to, wave);
                    else if constexpr (C < L) Q.template copy_one<C - P.N>(from_q, to + BP * 128, wave);
                });
            });
            now = next;
        }
        for (; t + 1 < t1; ++t) {
            const int next = now + 1 == R ? 0 : now + 1;
            half(first, reads, now, nothing);
            wait_vmcnt<0>();
            __syncthreads();
            if (t + R < t1) copy(t + R, now);
            half(second, reads, next, nothing);
            now = next;
        }
        half(first, reads, now, nothing);
        half(second, none, 0, nothing);
        static_for<0, FP>([&](auto I) __attribute__((always_inline)) { settle<(S::kAlone && I < FP - 1), I == 0>(acc[I]); });
    } else {
        // the chunks of a step are loaded two steps ahead (one: 24 us for 1531 x 1001 x 777 f16)
        auto load = [&](int t, auto X) __attribute__((always_inline)) {
            P.template load<X>(t * KE, wave, lane);
            Q.template load<X>(t * KE, wave, lane);
        };
        auto store = [&](auto X) __attribute__((always_inline)) {       // set and stage go by the step's parity
            P.template store<X>(lds + X * S::kStage, wave, lane);
            Q.template store<X>(lds + X * S::kStage + BP * 128, wave, lane);
        };
        auto step = [&](int t, auto X) __attribute__((always_inline)) { // a step of parity X
            constexpr std::integral_constant<int, 1 - X> other{};
            __syncthreads();
            if (t + 2 < t1) load(t + 2, X);
            read(X, first);
            read(X, second);
            products(first);
            products(second);
            if (t + 1 < t1) store(other);
        };
        if (t0 < t1) {
            load(t0, first);
            if (t0 + 1 < t1) load(t0 + 1, second);
            store(first);
        }
        for (int t = t0; t < t1; t += 2) {
            step(t, first);
            if (t + 1 < t1) step(t + 1, second);
        }
    }
    const int q0 = tq * BQ + wq, p0 = tp * BP + wp;
    Columns<T> columns;
    load_columns<T, Out, S::kPW>(a.e, p0, lane, columns);
    __syncthreads();                                // (the sums take the stages' place)
    float *sums = (float *)(lds + wave * S::kSums);
    const float *rows = sizeof(T) == 1 ? (const float *)(lds + S::kRows) + wq : nullptr;
    const int r = lane & 15, g = lane >> 4;
#pragma nounroll
    for (int h = 0; h < S::kQW / S::kSQ; ++h) {
        static_for<0, S::kQW / S::kSQ>([&](auto X) __attribute__((always_inline)) {
            if (X == h) {
#pragma unroll
                for (int j = 0; j < S::kSQ / 16; ++j)
#pragma unroll
                    for (int i = 0; i < FP; ++i) *(v4f *)(sums + (16 * j + r) * S::kSumsLd + 16 * i + 4 * g) = acc[i][X * (S::kSQ / 16) + j];
                // (unlike in either branch: or the last stores become one, from an address, and the sums go to memory for it)
                asm volatile("; part %0" ::"n"((int)X));
            }
        });
        __builtin_amdgcn_wave_barrier();
        epilogue<T, Out, sizeof(T) == 1 || !PK, S::kPW, S::kSQ>(a.e, partial, columns, sums, rows + h * S::kSQ, q0 + h * S::kSQ, p0, lane);
        __builtin_amdgcn_wave_barrier();
    }
}

template <class T, bool PK, bool QK, int BP, int BQ, int WP, int WQ, bool DIRECT, class Out>
__global__ __launch_bounds__(64 * WP * WQ) void product_kernel(Product a, float *partial, int steps_per_split, int tiles_p, int tiles_q, int blocks)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int block = (int)(blockIdx.z * kGridRow + blockIdx.x);
    if (block >= blocks) return;
    product_tile<T, Out, PK, QK, BP, BQ, WP, WQ, DIRECT>(a, partial, steps_per_split, tiles_p, tiles_q, block, lds);
}

// dx, dw and the bias gradient of a layer in one launch: each alone leaves compute units without work in its last round, or
// in its only one, and costs a launch (500 x 512 x 384 f32: the call 35 us in three launches, 19 in one with 64 x 64 tiles, 15 with 32 x 64; 1777 x 1024 x 2304 f16: 63
// and 33).
template <class T, int BP, int BQ>
__global__ __launch_bounds__(256) void product_pair_kernel(Product dx, Product dw, BiasGrad db, int blocks_dx, int blocks_dw, int blocks)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr int KE = 8 * Chunk<T>::E;
    int b = (int)(blockIdx.z * kGridRow + blockIdx.x);
    if (b >= blocks) return;
    if (b < blocks_dx) {
        product_tile<T, T, false, true, BP, BQ, 2, 2, true>(dx, nullptr, (dx.nk + KE - 1) / KE, (dx.e.np + BP - 1) / BP, (dx.e.nq + BQ - 1) / BQ, b, lds);
        return;
    }
    b -= (blocks_dx + 7) & ~7;                      // (the order of tiles goes by a work-group's XCD, its number modulo 8)
    if (b < 0) return;
    if (b < blocks_dw) {
        product_tile<T, T, false, false, BP, BQ, 2, 2, true>(dw, nullptr, (dw.nk + KE - 1) / KE, (dw.e.np + BP - 1) / BP, (dw.e.nq + BQ - 1) / BQ, b, lds);
        return;
    }
    bias_grad<T>(db, b - blocks_dw, (float *)lds);
}

// the sums of the parts, in their order, and the epilogue
template <class T, class Out>
__global__ __launch_bounds__(256) void product_join_kernel(Epilogue e, const float *partial, int splits)
{
    const int groups = (e.np + 7) / 8;
    const size_t at = ((size_t)blockIdx.y * kGridRow + blockIdx.x) * 256 + threadIdx.x;
    if (at >= (size_t)groups * e.nq) return;
    const int q = (int)(at / groups), p = (int)(at % groups) * 8;
    const size_t plane = (size_t)e.nq * groups * 8;
    const float *from = partial + (size_t)q * groups * 8 + p;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {                  // (their loads together: up to 16 parts wait once or twice)
        const v4f a = *(const v4f *)(from + s * plane), b = *(const v4f *)(from + s * plane + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = add_sums<T>(v[i], a[i]);
            v[4 + i] = add_sums<T>(v[4 + i], b[i]);
        }
    }
    finish_row<T, Out>(e, q, p, v);
}

template <class T, bool PK, bool QK, int BP, int BQ, int WP, int WQ, bool DIRECT, class Out>
hipError_t launch_product_shape(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    using S = ProductShape<T, BP, BQ, WP, WQ>;
    const int tiles_p = (a.e.np + BP - 1) / BP, tiles_q = (a.e.nq + BQ - 1) / BQ;
    const long long blocks = tile_order_blocks(tiles_q, tiles_p, false);
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const auto kernel = product_kernel<T, PK, QK, BP, BQ, WP, WQ, DIRECT, Out>;
    static std::atomic<unsigned long long> done{0};
    if (hipError_t e = allow_dynamic_lds((const void *)kernel, S::kLds, done)) return e;
    kernel<<<dim3(grid_row(blocks), plan.splits, grid_rows(blocks)), S::kThreads, S::kLds, st>>>(a, plan.splits > 1 ? partial : nullptr, plan.steps,
                                                                                                 tiles_p, tiles_q, (int)blocks);
    return hipGetLastError();
}

template <class T, bool PK, bool QK, class Out>
hipError_t launch_product_order(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    if (plan.direct) {
        if constexpr (sizeof(T) <= 2)
            if (plan.tile == 0) return launch_product_shape<T, PK, QK, 256, 256, 2, 2, true, Out>(a, plan, partial, st);
        if (plan.tile == 1) return launch_product_shape<T, PK, QK, 128, 128, 2, 2, true, Out>(a, plan, partial, st);
        return launch_product_shape<T, PK, QK, 64, 64, 2, 2, true, Out>(a, plan, partial, st);
    }
    if (plan.tile <= 1) return launch_product_shape<T, PK, QK, 128, 128, 2, 2, false, Out>(a, plan, partial, st);
    return launch_product_shape<T, PK, QK, 64, 64, 2, 2, false, Out>(a, plan, partial, st);
}

template <class T, class Out>
hipError_t launch_product_tiles(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    if constexpr (sizeof(T) == 1) return launch_product_order<T, true, true, Out>(a, plan, partial, st);
    else {
        if (a.p_k_rows && a.q_k_rows) return launch_product_order<T, true, true, Out>(a, plan, partial, st);
        if (a.q_k_rows) return launch_product_order<T, false, true, Out>(a, plan, partial, st);
        return launch_product_order<T, false, false, Out>(a, plan, partial, st);
    }
}

template <class T, class Out>
hipError_t launch_join(const Product &a, const ProductPlan &plan, const float *partial, hipStream_t st)
{
    const size_t threads = (size_t)a.e.nq * ((a.e.np + 7) / 8), groups = (threads + 255) / 256;
    if (groups > 0x7fffffff) return hipErrorInvalidValue;
    product_join_kernel<T, Out><<<dim3(grid_row(groups), grid_rows(groups)), 256, 0, st>>>(a.e, partial, plan.splits);
    return hipGetLastError();
}

// operands of type T, results, bias and residual of type Out
template <class T, class Out = T>
hipError_t launch_product_type(const Product &a, const ProductPlan &plan, float *partial, hipStream_t st)
{
    if (hipError_t e = plan.tile == kTileFew ? launch_few_tokens<T, Out>(a, plan, partial, st) : launch_product_tiles<T, Out>(a, plan, partial, st)) return e;
    return plan.splits > 1 ? launch_join<T, Out>(a, plan, partial, st) : hipSuccess;
}

template <class T, int BP, int BQ>
hipError_t launch_pair_shape(const Product &dx, const Product &dw, const BiasGrad &db, hipStream_t st)
{
    using S = ProductShape<T, BP, BQ, 2, 2>;
    const long long bx = tile_order_blocks((dx.e.nq + BQ - 1) / BQ, (dx.e.np + BP - 1) / BP, false);
    const long long bw = tile_order_blocks((dw.e.nq + BQ - 1) / BQ, (dw.e.np + BP - 1) / BP, false);
    const long long blocks = ((bx + 7) & ~7LL) + bw + bias_grad_blocks(db);
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    const auto kernel = product_pair_kernel<T, BP, BQ>;
    static std::atomic<unsigned long long> done{0};
    if (hipError_t e = allow_dynamic_lds((const void *)kernel, S::kLds, done)) return e;
    kernel<<<dim3(grid_row(blocks), 1, grid_rows(blocks)), S::kThreads, S::kLds, st>>>(dx, dw, db, (int)bx, (int)bw, (int)blocks);
    return hipGetLastError();
}

template <class T>
hipError_t launch_pair_type(const Product &dx, const Product &dw, const BiasGrad &db, int tile, hipStream_t st)
{
    if (tile == kTile128) return launch_pair_shape<T, 128, 128>(dx, dw, db, st);
    if constexpr (sizeof(T) == 4)
        if (tile == kTile32) return launch_pair_shape<T, 32, 64>(dx, dw, db, st);
    return launch_pair_shape<T, 64, 64>(dx, dw, db, st);
}

}  // namespace oz

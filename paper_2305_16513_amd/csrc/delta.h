// What the kernels of the gated delta rule share.
//
//   S_t = a_t S_{t-1} + k_t u_t^T,   u_t = beta_t (v_t - a_t S_{t-1}^T k_t),   o_t = scale S_t^T q_t,   a_t = exp(g_t)
//
// S is Dk x Dv.  Value head h reads queries and keys of head h / (Hv / Hk).
#pragma once
#include "seq.h"

namespace sws {

// Elements from one sequence, token, head to the next
struct Steps {
    int64_t batch, token, head;
};

struct DeltaArgs {
    int64_t B, T;
    int Hk, Hv, Dk, Dv;
    float scale;
    Steps q, k, v, g, beta, o;                        // o: of the output, or of its gradient
    int64_t pool;                                     // places of the states' pool
    const int *lengths, *slots;
};

// Tokens of sequence b that are there
__device__ __forceinline__ int64_t tokens_of(const DeltaArgs &a, int64_t b)
{
    const int64_t n = a.lengths ? a.lengths[b] : a.T;
    return n < 0 ? 0 : n < a.T ? n : a.T;
}

// exp(g) of a gate whose exp() is zero in fp32 is that of kLowest: sums of gates, and their differences, stay finite with -inf among them
constexpr float kLowest = -110.0f;

// A gate as it enters sums of gates.  (NaN stays NaN.)
__device__ __forceinline__ float gate(float g) { return g < kLowest ? kLowest : g; }

// ---- Chunks of 64 tokens on the matrix cores ----
//
// With G_i the sum of the chunk's gates up to token i, D_ij = exp(G_i - G_j) and S the state before the chunk:
//   A_ij = beta_i D_ij k_i.k_j (j < i),  P_ij = D_ij q_i.k_j (j <= i),  T = (I + A)^-1,
//   N = V - exp(G) K S,   U = T beta N,   O = scale (exp(G) Q S + P U),   S <- exp(G_63) S + K^T (exp(G_63 - G) U).
// All exponents are of sums of gates <= 0, so nothing overflows however strong the decay.  Tokens that are not there have beta = 0, g = 0 and
// rows of zeros: they change nothing.
//
// Where a number is not finite, zeros of T and P would carry it to earlier tokens.  Rows of T are then solved one by one, and forward products with T and P are done again
// without the rows of N or U that are not finite, and those behind them.
//
// Every product is of 16 x 16 tiles with a contraction of 32.  An operand is eight elements a lane: of row (or column) lane % 16 the
// contraction indices 4 g + e and 16 + 4 g + e (g = lane / 16, e = 0 .. 3) of a block of 32; the order of a contraction is free as long as both sides
// have the same.  This one is what two accumulator tiles hold (row 4 g + e of column lane % 16 each): a product becomes the
// next one's operand in its registers.
//
// 16-bit storage: elements of q, k, v, go enter as they are.  What has been computed (states, U, N, T, P ...) is fp32 and enters a product as pieces of the
// storage type: three in bf16, which together are the number; two in fp16, whose sum is off by 2^-22 of it, or 2^-25 where that is more (see scale_of).  So the fp32 outputs (states,
// gradients of gates) are as exact as fp32 products would leave them, and do not depend on whether a call's tokens are few or many; one piece
// would cost as much as the rounding of a 16-bit output, and the state's errors would add up over the chunks.  Products of pieces below the last piece's size
// are left out.  fp32: one piece, on the fp32 matrix instruction.
constexpr int kChunk = 64;

template <class E> struct Mx;
template <> struct Mx<__bf16> {
    typedef v8bf Frag;
    static constexpr int NP = 3;
    static __device__ __forceinline__ v4f mma(v4f c, Frag a, Frag b) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mx<_Float16> {
    typedef v8h Frag;
    static constexpr int NP = 2;
    static __device__ __forceinline__ v4f mma(v4f c, Frag a, Frag b) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mx<float> {
    typedef v8f_m Frag;
    static constexpr int NP = 1;
    static __device__ __forceinline__ v4f mma(v4f c, Frag a, Frag b)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};
template <class E> using Frag = typename Mx<E>::Frag;

// Two numbers as their pieces of 16 bits, the larger first, each pair a register.  An fp16 operand that is itself a product has to be one number for both its pieces: the
// compiler would take the upper one from an instruction that rounds the exact product to 16 bits, and subtract it from the product
// rounded to 32 bits first; next to a tie they are not the same.
template <class E>
__device__ __forceinline__ void pieces_of(float f, float g, unsigned (&p)[Mx<E>::NP])
{
    if constexpr (std::is_same_v<E, _Float16>) {
        typedef _Float16 v2h __attribute__((ext_vector_type(2)));
        asm("" : "+v"(f));
        asm("" : "+v"(g));
        const v2h h = {(_Float16)f, (_Float16)g};
        p[0] = __builtin_bit_cast(unsigned, h);
        p[1] = __builtin_bit_cast(unsigned, v2h{(_Float16)(f - (float)h[0]), (_Float16)(g - (float)h[1])});
    } else {
        // The first piece rounds to nearest, so that what is left has 16 bits at most and a sign of its own; the others cut these in two halves.
        typedef __bf16 v2b __attribute__((ext_vector_type(2)));
        p[0] = __builtin_bit_cast(unsigned, __builtin_convertvector((v2f{f, g}), v2b));
        asm("" : "+v"(p[0]));                         // (converted once, as a pair)
        f -= __uint_as_float(p[0] << 16);
        g -= __uint_as_float(p[0] & 0xffff0000u);
        auto upper = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u); };
        p[1] = upper(f, g);
        p[2] = upper(f - __uint_as_float(__float_as_uint(f) & 0xffff0000u), g - __uint_as_float(__float_as_uint(g) & 0xffff0000u));
    }
}

// Numbers of this magnitude and more have no finite pieces (fp16: what rounds to infinity; bf16: rounding the largest fp32 numbers up would, too)
template <class E> constexpr float kLimit = std::is_same_v<E, _Float16> ? 65520.0f : std::is_same_v<E, __bf16> ? 3.3895314e38f : __builtin_inff();

// A computed operand
template <class E> struct Pieces {
    Frag<E> p[Mx<E>::NP];
};

template <class E>
__device__ __forceinline__ Pieces<E> split(v4f a, v4f b)
{
    Pieces<E> r;
    if constexpr (Mx<E>::NP == 1) r.p[0] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    else {
        constexpr int NP = Mx<E>::NP;
        v4u u[NP];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            unsigned x[NP], y[NP];
            pieces_of<E>(a[2 * e], a[2 * e + 1], x);
            pieces_of<E>(b[2 * e], b[2 * e + 1], y);
#pragma unroll
            for (int n = 0; n < NP; ++n) u[n][e] = x[n], u[n][2 + e] = y[n];
        }
#pragma unroll
        for (int n = 0; n < NP; ++n) r.p[n] = __builtin_bit_cast(Frag<E>, u[n]);
    }
    return r;
}

// c + a b, the lesser products first
template <class E>
__device__ __forceinline__ v4f mma(v4f c, const Frag<E> &a, const Pieces<E> &b)
{
#pragma unroll
    for (int n = Mx<E>::NP - 1; n >= 0; --n) c = Mx<E>::mma(c, a, b.p[n]);
    return c;
}
template <class E>
__device__ __forceinline__ v4f mma(v4f c, const Pieces<E> &a, const Frag<E> &b)
{
#pragma unroll
    for (int n = Mx<E>::NP - 1; n >= 0; --n) c = Mx<E>::mma(c, a.p[n], b);
    return c;
}
template <class E>
__device__ __forceinline__ v4f mma(v4f c, const Pieces<E> &a, const Pieces<E> &b)
{
#pragma unroll
    for (int n = Mx<E>::NP - 1; n >= 0; --n)
#pragma unroll
        for (int i = 0; i <= n; ++i) c = Mx<E>::mma(c, a.p[i], b.p[n - i]);
    return c;
}

// Rows of W elements in LDS, and operands out of them.  Four elements of a row, a quad, stand together.
//   rows(p, t, kb)   lane's row is 16 t + lane % 16, the contraction index runs along it from 32 kb on
//   column(p, t, j)  the four elements of accumulator layout: rows 16 t + 4 g + e of column 16 j + lane % 16
//   cols(p, kb, j)   lane's column is 16 j + lane % 16, the contraction index is the row, 32 kb and on
//   column_of(p, t, j), cols_of(p, kb, j)   the same where j is not known to the compiler
// 16-bit types: column() is the transposing load, to which sixteen lanes point out four rows of four quads.  Rows have no gaps; the quad that belongs at c of row
// r stands at c ^ turn(r), so that both reads, of 16 rows x two quads and of 8 rows x four quads by half a wavefront, meet every bank
// once, and two neighbouring quads stay one 16-byte unit.  fp32: rows four elements apart.
template <class E, int W> struct Tile {
    static_assert(W == 16 || W == 32 || W == 64 || W == 128, "");
    static constexpr int KB = W / 32, KT = W / 16, LD = W;
    static constexpr int size(int rows) { return rows * LD; }
    static __device__ __forceinline__ int turn(int r)
    {
        return W == 128 ? 4 * (r & 7) + 2 * (r >> 3 & 1) : W == 64 ? 4 * (r >> 1 & 3) + 2 * (r >> 3 & 1) : W == 32 ? 4 * (r >> 2 & 1) + 2 * (r >> 3 & 1) : 0;
    }
    static __device__ __forceinline__ int at(int r, int quad) { return r * LD + 4 * (quad ^ turn(r)); }
    int row[KB ? KB : 1][2], col[KT];                 // this lane's elements of the first 16 rows

    __device__ __forceinline__ Tile(int tid = threadIdx.x)
    {
        const int l = tid % 16, g = tid % kWave / 16;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int half = 0; half < 2; ++half) row[kb][half] = at(l, 8 * kb + 4 * half + g);
#pragma unroll
        for (int j = 0; j < KT; ++j) col[j] = at(4 * g + l / 4, 4 * j + l % 4);
    }
    __device__ __forceinline__ Frag<E> rows(const E *p, int t, int kb) const
    {
        typedef typename Vec<E>::v4 V4;
        const V4 a = *(const V4 *)(p + 16 * LD * t + row[kb][0]), b = *(const V4 *)(p + 16 * LD * t + row[kb][1]);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ typename Vec<E>::v4 transposed(const E *p)
    {
        typedef __attribute__((address_space(3))) v4s lds_v4s;
        return __builtin_bit_cast(typename Vec<E>::v4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)p));
    }
    __device__ __forceinline__ typename Vec<E>::v4 column(const E *p, int t, int j) const { return transposed(p + 16 * LD * t + col[j]); }
    static __device__ __forceinline__ typename Vec<E>::v4 column_of(const E *p, int t, int j, int tid = threadIdx.x)
    {
        const int l = tid % 16, g = tid % kWave / 16;
        return transposed(p + 16 * LD * t + at(4 * g + l / 4, 4 * j + l % 4));
    }
    static __device__ __forceinline__ Frag<E> cols_of(const E *p, int kb, int j, int tid = threadIdx.x)
    {
        const auto a = column_of(p, 2 * kb, j, tid), b = column_of(p, 2 * kb + 1, j, tid);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ Frag<E> cols(const E *p, int kb, int j) const
    {
        const auto a = column(p, 2 * kb, j), b = column(p, 2 * kb + 1, j);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};
template <int W> struct Tile<float, W> {
    __device__ __forceinline__ Tile(int = 0) {}
    static constexpr int LD = W + 4;
    static constexpr int size(int rows) { return rows * LD; }
    static __device__ __forceinline__ int at(int r, int quad) { return r * LD + 4 * quad; }
    __device__ __forceinline__ v8f_m rows(const float *p, int t, int kb) const
    {
        const float *q = p + (16 * t + threadIdx.x % 16) * LD + 32 * kb + 4 * (threadIdx.x % kWave / 16);
        return __builtin_shufflevector(*(const v4f *)q, *(const v4f *)(q + 16), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ v4f column(const float *p, int t, int j) const
    {
        const float *q = p + (16 * t + 4 * (threadIdx.x % kWave / 16)) * LD + 16 * j + threadIdx.x % 16;
        return v4f{q[0], q[LD], q[2 * LD], q[3 * LD]};
    }
    __device__ __forceinline__ v8f_m cols(const float *p, int kb, int j) const
    {
        return __builtin_shufflevector(column(p, 2 * kb, j), column(p, 2 * kb + 1, j), 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ v4f column_of(const float *p, int t, int j, int = 0) const { return column(p, t, j); }
    __device__ __forceinline__ v8f_m cols_of(const float *p, int kb, int j, int = 0) const { return cols(p, kb, j); }
};

template <class V4>
__device__ __forceinline__ v4f widen(V4 v)
{
    return v4f{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}

// exp(x), x <= 0: the storage's precision at least
template <class E>
__device__ __forceinline__ float decay(float x)
{
    if constexpr (sizeof(E) == 4) return expf(x);
    else return __expf(x);
}

// Up to 64 rows of `width` <= W elements, `step` apart, as 16-byte units in registers of NT threads; rows from n on and elements from
// width on are zeros.  FULL: width = W, every row begins at a multiple of 16 bytes, and step is W at least and below 2^22: rows from n on
// lie behind the end of a buffer, which loads nothing there.
template <class E, int W, int NT, bool FULL> struct Rows {
    static constexpr int PER = 16 / (int)sizeof(E), UNITS = W / PER, N = (kChunk * UNITS + NT - 1) / NT;
    static_assert(kChunk * UNITS % NT == 0 && NT % UNITS == 0, "whole rounds of whole rows");
    v4u r[N];

    __device__ __forceinline__ void load(const E *p, int64_t step, int n, int width, int tid)
    {
        if constexpr (FULL) {
            const int st = (int)step * (int)sizeof(E);
            const __amdgpu_buffer_rsrc_t from = rsrc(p, n > 0 ? (unsigned)((n - 1) * st + W * (int)sizeof(E)) : 0u);
            int at = tid / UNITS * st + tid % UNITS * 16;
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(from, at + i * (NT / UNITS) * st, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int u = tid + i * NT, row = u / UNITS, c = u % UNITS * PER;
                const E *q = p + row * step + c;
                typedef E VP __attribute__((ext_vector_type(16 / sizeof(E))));
                VP v;
#pragma unroll
                for (int e = 0; e < PER; ++e) v[e] = row < n && c + e < width ? q[e] : (E)0.0f;
                r[i] = __builtin_bit_cast(v4u, v);
            }
        }
    }
    // to a tile in LDS
    __device__ __forceinline__ void store(E *to, int tid) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = tid + i * NT, row = u / UNITS, c = u % UNITS;
            if constexpr (sizeof(E) == 2) *(v4u *)(to + Tile<E, W>::at(row, 2 * c)) = r[i];
            else *(v4u *)(to + Tile<E, W>::at(row, c)) = r[i];
        }
    }
};

// Where the operands of the triangular matrices lie in the workspace, in the order in which lanes take them: per tile row rt of T or P the blocks of 32
// columns up to the diagonal, of their transposes those from it on.
__device__ __forceinline__ constexpr int lower_at(int rt, int kb) { return rt < 2 ? rt : 2 + (rt - 2) * 2 + kb; }
__device__ __forceinline__ constexpr int upper_at(int rt, int kb) { return rt < 2 ? rt * 2 + kb : 2 + rt; }
constexpr int kFrags = 6;

// Bytes of one of T, P, their transposes; of the chunk's factors (exp(G), exp(G_63 - G), beta: 64 floats each)
template <class E> constexpr int tri_bytes() { return kFrags * Mx<E>::NP * kWave * 8 * (int)sizeof(E); }
constexpr int kFactorBytes = 3 * kChunk * 4;

// A computed operand to and from memory, in the order in which lanes hold it: operand `at` of an array
template <class E>
__device__ __forceinline__ void put_pieces(E *to, int at, const Pieces<E> &p, int tid = threadIdx.x)
{
#pragma unroll
    for (int n = 0; n < Mx<E>::NP; ++n) *(Frag<E> *)(to + ((at * Mx<E>::NP + n) * kWave + tid % kWave) * 8) = p.p[n];
}
template <class E>
__device__ __forceinline__ Pieces<E> get_pieces(const E *from, int at, int tid = threadIdx.x)
{
    Pieces<E> p;
#pragma unroll
    for (int n = 0; n < Mx<E>::NP; ++n) p.p[n] = *(const Frag<E> *)(from + ((at * Mx<E>::NP + n) * kWave + tid % kWave) * 8);
    return p;
}

// What the passes from chunk to chunk leave for the gradients, in fp32, per chunk and 16 columns of the state: S (or the gradient of the state behind
// the chunk) as DK / 32 operands whose contraction index is the key's element, U (or dR) as two whose contraction index is the token; every operand
// as two units of 16 bytes a lane.  The gradients lay these down in LDS in pieces, UNITS units of 16 bytes a lane (fp32: as they are), and need the operands whose
// contraction index is the column of the state.
template <class E> struct Kept {
    static constexpr int UNITS = Mx<E>::NP == 1 ? 2 : Mx<E>::NP, OPERAND = 1024 * UNITS;      // bytes of one in LDS
    static constexpr int64_t state(int DK) { return (int64_t)DK / 32 * 2048; }    // bytes in memory
    static constexpr int64_t rows() { return 2 * 2048; }
    static __device__ __forceinline__ int place(int g, int r) { return (16 * g + (r ^ 4 * g)) * 16; }

    static __device__ __forceinline__ void put(char *to, int kb, v4f a, v4f b)
    {
        char *const q = to + 2048 * kb + place(threadIdx.x % kWave / 16, threadIdx.x % 16);
        *(v4f *)q = a;
        *(v4f *)(q + 1024) = b;
    }
    // A lane's two units of an operand, lanes in the order of the units, from memory (`from` is the wavefront's); and to LDS
    static __device__ __forceinline__ void load(const char *from, int lane, v4f (&u)[2])
    {
        const __amdgpu_buffer_rsrc_t b = rsrc(from, 2048);
        u[0] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(b, 16 * lane, 0, 0));
        u[1] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(b, 16 * lane + 1024, 0, 0));
    }
    static __device__ __forceinline__ void lay(char *to, int at, int lane, const v4f (&u)[2])
    {
        char *const q = to + OPERAND * at + 16 * lane;
        if constexpr (Mx<E>::NP == 1) {
            *(v4f *)q = u[0];
            *(v4f *)(q + 1024) = u[1];
        } else {
            const Pieces<E> p = split<E>(u[0], u[1]);
#pragma unroll
            for (int n = 0; n < UNITS; ++n) *(Frag<E> *)(q + 1024 * n) = p.p[n];
        }
    }
    // Of two groups of 16 columns in LDS, `group` bytes apart: lane's element (of the key, or token) is 16 j + lane % 16, the contraction index is the column.
    static __device__ __forceinline__ Pieces<E> columns(const char *p, int group, int j, int tid = threadIdx.x)
    {
        const int l = tid % 16, g = tid % kWave / 16;
        Pieces<E> r;
        if constexpr (Mx<E>::NP > 1) {
            const char *const q = p + place(l % 4, 4 * g + l / 4) + OPERAND * (j >> 1) + 8 * (j & 1);
#pragma unroll
            for (int n = 0; n < UNITS; ++n) {
                const auto a = Tile<E, 32>::transposed((const E *)(q + 1024 * n)), b = Tile<E, 32>::transposed((const E *)(q + group + 1024 * n));
                r.p[n] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        } else {
            const char *const q = p + OPERAND * (j >> 1) + 1024 * (j & 1) + 4 * (l % 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) r.p[0][e] = *(const float *)(q + (e < 4 ? 0 : group) + place(l / 4, 4 * g + (e & 3)));
        }
        return r;
    }
    // The same of both j = 2 m and 2 m + 1, the two halves of every unit.  One of them would leave half of the banks idle: every second sixteen lanes take the
    // other one first.
    static __device__ __forceinline__ void both(const char *p, int group, int m, Pieces<E> (&r)[2], int tid = threadIdx.x)
    {
        if constexpr (Mx<E>::NP > 1) {
            const int l = tid % 16, g = tid % kWave / 16, odd = 8 * (g & 1);
            const char *const q = p + place(l % 4, 4 * g + l / 4) + OPERAND * m;
#pragma unroll
            for (int n = 0; n < UNITS; ++n) {
                typename Vec<E>::v4 x[2][2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const auto a = Tile<E, 32>::transposed((const E *)(q + group * t + 1024 * n + odd));
                    const auto b = Tile<E, 32>::transposed((const E *)(q + group * t + 1024 * n + (8 - odd)));
                    const v2u u = __builtin_bit_cast(v2u, a), v = __builtin_bit_cast(v2u, b);
                    x[0][t] = __builtin_bit_cast(typename Vec<E>::v4, odd ? v : u);
                    x[1][t] = __builtin_bit_cast(typename Vec<E>::v4, odd ? u : v);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) r[h].p[n] = __builtin_shufflevector(x[h][0], x[h][1], 0, 1, 2, 3, 4, 5, 6, 7);
            }
        } else {
            r[0] = columns(p, group, 2 * m, tid);
            r[1] = columns(p, group, 2 * m + 1, tid);
        }
    }
};

// fp16 numbers reach from 2^-24 to 65504; states and corrections are as large as the values that they are made of.  They are linear in the values and the state before the
// first token, and backward in the gradients of the outputs and of the last state.  So a value head's passes work on these times a power of two and take it back
// in what they give.  It brings the largest of them to 4 .. 8 if it is below (else a loss that is a mean over tokens would leave its gradients where the
// pieces have few bits), to 128 .. 256 if it is beyond (a state may then grow 256-fold), and is 1 between: bits that are worth 2^-25 are worth that of numbers of that size.
// Numbers that are not finite do not count.
template <class E> constexpr bool kScaled = std::is_same_v<E, _Float16>;

// The power of two for a largest magnitude, given as its fp32 bits
__device__ __forceinline__ float scale_of(unsigned top)
{
    const int at = (int)(top >> 23) - 127, by = at < 2 ? 2 - at : at < 8 ? 0 : 7 - at, e = by < -100 ? -100 : by > 100 ? 100 : by;
    return top ? __uint_as_float((unsigned)(127 + e) << 23) : 1.0f;
}

// A magnitude's bits, 0 where it is not finite
__device__ __forceinline__ unsigned magnitude(float f)
{
    const unsigned u = __float_as_uint(f) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

__device__ __forceinline__ unsigned max_lanes(unsigned v)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const unsigned t = (unsigned)__shfl_xor((int)v, d);
        v = v > t ? v : t;
    }
    return v;
}

// The largest magnitudes of each chunk, two numbers a chunk (of the values, and with the first chunk the state; of the outputs' gradients, and the last state's); of which
// a wavefront makes the scale of all of a sequence's
__device__ __forceinline__ float scale_over(const unsigned *tops, int chunks, int which)
{
    unsigned top = 0;
    for (int c = threadIdx.x % kWave; c < chunks; c += kWave) top = top > tops[2 * c + which] ? top : tops[2 * c + which];
    return scale_of((unsigned)__builtin_amdgcn_readfirstlane((int)max_lanes(top)));
}

// What the first pass needs for that (go, gstate: gradients only)
struct Magnitudes {
    const void *v, *go;
    const float *state, *gstate;
    unsigned *tops;
};

// The passes from chunk to chunk: outputs; states and U for the gradients; the backward pass
enum ScanMode { FORWARD, KEEP, BACKWARD };

struct ScanWs {
    const char *tri;                                  // per chunk T beta and P, or T beta, T^T and P^T
    const float *factors;
    void *u, *s;                                      // KEEP: U and the states before the chunks; BACKWARD: dR and the gradients of those behind
    const unsigned *tops;                             // fp16: magnitudes per chunk
    float *scales;                                    // fp16: per value head the scale of U and S, and that of dR and dS, for the gradients
    int chunks, cols;                                 // of a sequence; of the state as it is kept (a multiple of 32)
};

// Whether rows of W elements can be loaded by Rows<FULL>
template <class E>
bool full_rows(const Steps &s, int W, const void *p)
{
    constexpr int PER = 16 / (int)sizeof(E);
    return s.batch % PER == 0 && s.token % PER == 0 && s.head % PER == 0 && s.token >= W && s.token < 1 << 22 && sixteen({p});
}

__device__ __forceinline__ int chunks_of(int64_t tokens) { return (int)((tokens + kChunk - 1) / kChunk); }

}  // namespace sws

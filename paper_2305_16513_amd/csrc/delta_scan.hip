// The passes of the gated delta rule that go from chunk to chunk, on 16-bit storage: forward with the outputs, forward leaving what the gradients
// need, and backward.
//
// Columns of the state do not meet: 16 of them, Dk x 16 floats in accumulator layout, are one wavefront's, which takes its sequence's chunks
// one after the other.  Per chunk
//     N = V - exp(G) K S,   U = T beta N,   S <- exp(G_63) S + K^T (exp(G_63 - G) U),   O = scale (exp(G) Q S + P U)
// and S, N and U go from one product into the next in registers (see delta.h).  Backward, with dS the gradient of the state behind the chunk:
//     dU = scale P^T dO + exp(G_63 - G) (K dS),   dR = T^T dU,   dS <- exp(G_63) dS + scale Q^T (exp(G) dO) - K^T (beta exp(G) dR)
//
// Bound by the length of that chain, chunk after chunk: reads of LDS, products and the splitting of their results, one after the other, not by the rate of
// any.  What is not part of it is done by others.  T and P are another kernel's, for all chunks at once.  The 16 columns are two wavefronts', each
// half of the state's rows; they exchange their halves of K S once per chunk, and both take N and U.  Two more compute, forward, O, a
// chunk behind, from the operands of S and the accumulators of U that the first ones leave in LDS; backward, a chunk ahead, the terms with dO, which do not
// depend on dS, and leave them as accumulators; each half of the tokens.  Four load the chunks to come and stage K, Q, V, T in LDS.  All meet
// twice per chunk.  O is computed transposed, so that a lane has four neighbouring elements of a token.  A workgroup has NS = 2 groups of 16 columns, or one where
// there are too few states to give every CU two.
//
// bf16, Dk = Dv = 128: one sequence of 16384 tokens, 32 states: 551 us, 256 chunks of 4500 cycles one after the other, in which a wavefront of the states issues 84 matrix
// instructions (1340 cycles) and some 440 vector ones (1770), 264 of them to cut S, N and U into three pieces.  Counters: vector units 32 % of the
// time, matrix units 22 %, LDS 59 %.  Four sequences of 4096, 16 states each: forward 199 us (47, 34 and 69 %); leaving states 179 us, backward 234 us (616 and 759 MB with what
// the gradients need: 120 and 148 us of HBM).
#include "delta.h"

namespace sws {

namespace {

// Wavefronts: of the states, of the terms beside them (not where only states are wanted), two that load K and V (dO), two that load T, the factors and Q
constexpr int scan_threads(int NS, int MODE) { return kWave * ((MODE == KEEP ? 2 * NS : 4 * NS) + 4); }

// The workgroup's LDS: two of K, Q, V (or dO) and the chunk's factors, T (or T^T); what goes from the wavefronts of the states to those
// beside them, or back: forward the operands of S, and two of U; backward two of scale Q^T (exp(G) dO) and of scale P^T dO, as accumulators; the halves of K S.
template <class E, int DK, int NS, int MODE>
struct ScanLds {
    static constexpr int XS = MODE == FORWARD ? DK / 32 * Mx<E>::NP * kWave : DK / 16 * kWave, XU = 4 * kWave;
    static constexpr bool QUERIES = MODE != KEEP;
    v4f xs[MODE == BACKWARD ? 2 : 1][QUERIES ? NS * XS : 1], xu[QUERIES ? 2 : 1][QUERIES ? NS * XU : 1];
    v4f half[2][NS][4 * kWave];
    E ks[2][kChunk * DK], qs[QUERIES ? 2 : 1][QUERIES ? kChunk * DK : 8];
    v4u ts[tri_bytes<E>() / 16];
    E vs[2][kChunk * 16 * NS];
    float fs[2][4 * kChunk];                          // (three of 64; the last is nobody's)
};

// Where the operand of tile row t and block kb of a triangular matrix is, -1: there is none.  Of its blocks one has four operands, the other two.
template <bool UPPER> __device__ __forceinline__ constexpr int tri_at(int t, int kb)
{
    return UPPER ? (kb >= t / 2 ? upper_at(t, kb) : -1) : kb <= t / 2 ? lower_at(t, kb) : -1;
}

// x[t] += M_t,kb a over one block of a triangular matrix; the products of one accumulator as far apart as there are tiles
template <class E, bool UPPER>
__device__ __forceinline__ void tri_mul(v4f (&x)[4], const Pieces<E> (&m)[kFrags], const Pieces<E> &a, int kb)
{
#pragma unroll
    for (int n = Mx<E>::NP - 1; n >= 0; --n)          // the lesser products first
#pragma unroll
        for (int i = 0; i <= n; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (tri_at<UPPER>(t, kb) >= 0) x[t] = Mx<E>::mma(x[t], m[tri_at<UPPER>(t, kb)].p[i], a.p[n - i]);
}

// (Wavefronts per SIMD: the compiler sees no LDS; below half of the registers accumulators are ordinary ones and need no moves.)
template <class E, int DK, int NS, int MODE, bool FULL>
__global__ __launch_bounds__(scan_threads(NS, MODE)) __attribute__((amdgpu_waves_per_eu(NS == 2 && MODE != KEEP ? 3 : 2)))
void delta_scan_kernel(const E *__restrict__ q, const E *__restrict__ k, const E *__restrict__ v, E *__restrict__ o, float *__restrict__ state,
                       ScanWs ws, DeltaArgs a)
{
    constexpr int NL = 128, NP = Mx<E>::NP, W = 16 * NS, TRI = tri_bytes<E>(), KB = DK / 32, KT = DK / 16, HB = KB / 2, HT = KT / 2;
    constexpr int KINDS = MODE == FORWARD ? 2 : 3, T_AT = MODE == BACKWARD ? 1 : 0, P_AT = MODE == BACKWARD ? 2 : 1;
    typedef ScanLds<E, DK, NS, MODE> Lds;
    typedef Tile<E, DK> Keys;
    constexpr bool QUERIES = Lds::QUERIES;
    constexpr int XS = Lds::XS, XU = Lds::XU;
    extern __shared__ __align__(16) char lds[];
    Lds &m = *(Lds *)lds;
    auto &ks = m.ks;
    auto &qs = m.qs;
    auto &vs = m.vs;
    auto &xs = m.xs;
    auto &xu = m.xu;
    auto &fs = m.fs;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), w = wave % NS, hf = wave / NS % 2, lane = threadIdx.x % kWave, l = lane % 16,
              gr = lane / 16;
    const int64_t head = group_of(), b = group_of() / (unsigned)a.Hv;
    if (b >= a.B) return;
    const int h = (int)(head - b * a.Hv), hk = h / (a.Hv / a.Hk);
    const int col0 = blockIdx.y * W;                  // the workgroup's first column of the state
    int64_t len = tokens_of(a, b);
    const int64_t slot = a.slots ? a.slots[b] : b;
    if (state && a.slots && (slot < 0 || slot >= a.pool)) len = 0;
    const int chunks = chunks_of(len);
    const int first = MODE == BACKWARD ? chunks - 1 : 0, step = MODE == BACKWARD ? -1 : 1;   // the i-th chunk is first + i * step
    // (the last product's rounding is to the storage type, or fp32: the scale and its inverse are powers of two)
    const float rise = kScaled<E> && wave < (MODE == KEEP ? 2 : 4) * NS ? scale_over(ws.tops + 2 * head * ws.chunks, chunks, MODE == BACKWARD) : 1.0f, fall = 1.0f / rise;
    auto barrier = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    auto tri_of = [&](int i, int kind) {
        return (const E *)(ws.tri + (head * ws.chunks + first + i * step) * (int64_t)(KINDS * TRI) + kind * TRI);
    };
    // This wavefront's half of the keys' elements in LDS: operands of rows, of columns
    int row[HB][2], col[HT];
#pragma unroll
    for (int kb = 0; kb < HB; ++kb)
#pragma unroll
        for (int n = 0; n < 2; ++n) row[kb][n] = Keys::at(l, 8 * (HB * hf + kb) + 4 * n + gr);
#pragma unroll
    for (int j = 0; j < HT; ++j) col[j] = Keys::at(4 * gr + l / 4, 4 * (HT * hf + j) + l % 4);
    auto rows = [&](const E *p, int t, int kb) {
        typedef typename Vec<E>::v4 V4;
        const V4 x = *(const V4 *)(p + 16 * DK * t + row[kb][0]), y = *(const V4 *)(p + 16 * DK * t + row[kb][1]);
        return Frag<E>(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto cols = [&](const E *p, int kb, int j) {
        const auto x = Keys::transposed(p + 32 * DK * kb + col[j]), y = Keys::transposed(p + 32 * DK * kb + 16 * DK + col[j]);
        return Frag<E>(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const v4f zero = {0, 0, 0, 0};
    // Of accumulators whose rows are tokens: the least of a column's numbers, and its rows from `first` on replaced
    auto least_of_columns = [&](int first) {
#pragma unroll
        for (int d = 16; d < kWave; d *= 2) {
            const int other = __shfl_xor(first, d);
            first = first < other ? first : other;
        }
        return first;
    };
    auto keep_before = [&](v4f (&x)[4], int first, float by) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * t + 4 * gr + e >= first) x[t][e] = by;
    };

    if (wave < 2 * NS) {
        float *const sp = state && (len > 0 || MODE == BACKWARD) ? state + (slot * a.Hv + h) * (int64_t)a.Dk * a.Dv : nullptr;
        v4f s[HT];
        auto each = [&](auto &&f) {                   // f(element, its place in the state) of this lane's that are there
            int t = threadIdx.x;
            asm volatile("" : "+v"(t));               // (the places are not kept in registers until the end)
            const int my = col0 + 16 * w + t % 16;    // this lane's column
#pragma unroll
            for (int i = 0; i < HT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 16 * (HT * hf + i) + 4 * (t % kWave / 16) + e;
                    if (r < a.Dk && my < a.Dv) f(i, e, r * a.Dv + my);
                }
        };
#pragma unroll
        for (int i = 0; i < HT; ++i) s[i] = zero;
        if (sp) each([&](int i, int e, int at) { s[i][e] = kScaled<E> ? rise * sp[at] : sp[at]; });
        if (kScaled<E> && MODE != FORWARD && blockIdx.y == 0 && threadIdx.x == 0 && chunks > 0) ws.scales[2 * head + (MODE == BACKWARD)] = rise;
        Pieces<E> sx[HB];
#pragma unroll
        for (int kb = 0; kb < HB; ++kb) {
            sx[kb] = split<E>(s[2 * kb], s[2 * kb + 1]);
            if constexpr (MODE == FORWARD) put_pieces<E>((E *)(xs[0] + w * XS), HB * hf + kb, sx[kb]);
        }
        barrier();
        if constexpr (MODE == BACKWARD) barrier();
        for (int i = 0; i < chunks; ++i) {
            const int p = i & 1;
            const E *const kc = ks[p];
            const float *const fc = fs[p];
            const int64_t kept = (head * ws.chunks + first + i * step) * (ws.cols / 16) + (col0 / 16 + w);
            char *const up = (char *)ws.u + kept * Kept<E>::rows();
            if constexpr (MODE != FORWARD) {
                char *const to = (char *)ws.s + kept * Kept<E>::state(DK);
#pragma unroll
                for (int kb = 0; kb < HB; ++kb) Kept<E>::put(to, HB * hf + kb, s[2 * kb], s[2 * kb + 1]);
            }
            auto factor = [&](int which, int t) { return *(const v4f *)(fc + which * kChunk + 16 * t + 4 * gr); };
            // Everything that is read of K for one product goes out in one go, and is taken as it comes: a read takes as long as eight products.
            Frag<E> kf[HB][4];
            v4f x[4], f0[4], f1[4];                   // K S: rows are tokens
            typename Vec<E>::v4 vt[4];
#pragma unroll
            for (int kb = 0; kb < HB; ++kb)
#pragma unroll
                for (int t = 0; t < 4; ++t) kf[kb][t] = rows(kc, t, kb);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = zero;
#pragma unroll
            for (int kb = 0; kb < HB; ++kb)
#pragma unroll
                for (int n = NP - 1; n >= 0; --n)
#pragma unroll
                    for (int t = 0; t < 4; ++t) x[t] = Mx<E>::mma(x[t], kf[kb][t], sx[kb].p[n]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                m.half[hf][w][t * kWave + lane] = x[t];
                f0[t] = factor(MODE == BACKWARD ? 1 : 0, t);
                if constexpr (MODE != BACKWARD) vt[t] = Tile<E, W>::column_of(vs[p], t, w);
            }
            barrier();
            Pieces<E> tf[kFrags];
            Frag<E> cf[HT][2];
#pragma unroll
            for (int t = 0; t < 4; ++t) f1[t] = m.half[hf ^ 1][w][t * kWave + lane];
            // (T's larger block; the other one when K S, V and the factors have been used)
            constexpr bool UPPER = MODE == BACKWARD;
            auto tri_read = [&](int kb) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (tri_at<UPPER>(t, kb) >= 0) tf[tri_at<UPPER>(t, kb)] = get_pieces<E>((const E *)m.ts, tri_at<UPPER>(t, kb));
            };
            tri_read(UPPER);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][e] = hf ? f1[t][e] + x[t][e] : x[t][e] + f1[t][e];      // (the same sum in both)
            const float all = fc[kChunk - 1];         // exp(G_63)
            Pieces<E> d0, d1;
            if constexpr (MODE != BACKWARD) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {         // N
                    const v4f v4 = widen(vt[t]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][e] = (kScaled<E> ? rise * v4[e] : v4[e]) - f0[t][e] * x[t][e];
                }
                const Pieces<E> n0 = split<E>(x[0], x[1]), n1 = split<E>(x[2], x[3]);
                tri_read(1);
#pragma unroll
                for (int t = 0; t < 4; ++t) x[t] = zero;
                tri_mul<E, false>(x, tf, n0, 0);
                tri_mul<E, false>(x, tf, n1, 1);
                if (MODE == FORWARD && __builtin_expect(__any(x[3][0] != x[3][0]), 0)) {
                    // A row of N that is not finite has reached all rows of U, times zeros of T, in its column.  Again without it and the rows behind it, which are then not finite.
                    // (All of N is still in LDS.)
                    int first = kChunk;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const v4f a0 = m.half[0][w][t * kWave + lane], a1 = m.half[1][w][t * kWave + lane], gm = factor(0, t), v4 = widen(Tile<E, W>::column_of(vs[p], t, w));
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[t][e] = (kScaled<E> ? rise * v4[e] : v4[e]) - gm[e] * (a0[e] + a1[e]);
                            const int row = 16 * t + 4 * gr + e;
                            if (!(__builtin_fabsf(x[t][e]) < kLimit<E>)) first = first < row ? first : row;
                        }
                    }
                    first = least_of_columns(first);
                    keep_before(x, first, 0.0f);
                    const Pieces<E> m0 = split<E>(x[0], x[1]), m1 = split<E>(x[2], x[3]);
                    tri_read(0);
                    tri_read(1);
#pragma unroll
                    for (int t = 0; t < 4; ++t) x[t] = zero;
                    tri_mul<E, false>(x, tf, m0, 0);
                    tri_mul<E, false>(x, tf, m1, 1);
                    keep_before(x, first, __builtin_nanf(""));
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) f1[t] = factor(1, t);
#pragma unroll
                for (int j = 0; j < HT; ++j) {
                    cf[j][0] = cols(kc, 0, j);
                    cf[j][1] = cols(kc, 1, j);
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (MODE == KEEP) Kept<E>::put(up, hf, hf ? x[2] : x[0], hf ? x[3] : x[1]);
                else {
                    v4f *const to = xu[p] + w * XU + 2 * hf * kWave + lane;
                    to[0] = hf ? x[2] : x[0];
                    to[kWave] = hf ? x[3] : x[1];
                }
            } else {
                const v4f *const zc = xu[p] + w * XU + lane;
#pragma unroll
                for (int t = 0; t < 4; ++t) {         // dU
                    const v4f z = zc[t * kWave];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][e] = f0[t][e] * x[t][e] + z[e];
                    const v4f gm = factor(0, t), bt = factor(2, t);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f1[t][e] = -gm[e] * bt[e];
                }
                const Pieces<E> u0 = split<E>(x[0], x[1]), u1 = split<E>(x[2], x[3]);
                tri_read(0);
#pragma unroll
                for (int t = 0; t < 4; ++t) x[t] = zero;
                tri_mul<E, true>(x, tf, u1, 1);
                tri_mul<E, true>(x, tf, u0, 0);
#pragma unroll
                for (int j = 0; j < HT; ++j) {
                    cf[j][0] = cols(kc, 0, j);
                    cf[j][1] = cols(kc, 1, j);
                }
                __builtin_amdgcn_sched_barrier(0);
                Kept<E>::put(up, hf, hf ? x[2] : x[0], hf ? x[3] : x[1]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][e] *= f1[t][e];
            d0 = split<E>(x[0], x[1]), d1 = split<E>(x[2], x[3]);
            const v4f *const yc = xs[QUERIES ? p : 0] + w * XS + HT * hf * kWave + lane;
#pragma unroll
            for (int j = 0; j < HT; ++j) {
                if constexpr (MODE == BACKWARD) {
                    const v4f y = yc[j * kWave];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] = all * s[j][e] + y[e];
                } else
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] *= all;
            }
#pragma unroll
            for (int n = NP - 1; n >= 0; --n) {
#pragma unroll
                for (int j = 0; j < HT; ++j) s[j] = Mx<E>::mma(s[j], cf[j][0], d0.p[n]);
#pragma unroll
                for (int j = 0; j < HT; ++j) s[j] = Mx<E>::mma(s[j], cf[j][1], d1.p[n]);
            }
#pragma unroll
            for (int kb = 0; kb < HB; ++kb) {
                sx[kb] = split<E>(s[2 * kb], s[2 * kb + 1]);
                if constexpr (MODE == FORWARD) put_pieces<E>((E *)(xs[0] + w * XS), HB * hf + kb, sx[kb]);      // (the last ones have been read)
            }
            barrier();
        }
        if (MODE != KEEP && sp) each([&](int i, int e, int at) { sp[at] = kScaled<E> ? fall * s[i][e] : s[i][e]; });
        return;
    }

    if (MODE != KEEP && wave < 4 * NS) {              // beside the states: tokens of tiles hf and 3 - hf
        const int tile[2] = {hf, 3 - hf};
        const float scale = !kScaled<E> ? a.scale : a.scale * (MODE == FORWARD ? fall : rise);
        Pieces<E> pf[3];                              // of P: one block of the first and two of the other; of P^T: two and one
        auto fetch = [&](int i) {
            const E *const t = tri_of(i, P_AT);
            if constexpr (MODE == FORWARD) {
                pf[0] = get_pieces<E>(t, hf);
                pf[1] = get_pieces<E>(t, 4 - 2 * hf);
                pf[2] = get_pieces<E>(t, 5 - 2 * hf);
            } else {
                pf[0] = get_pieces<E>(t, 2 * hf);
                pf[1] = get_pieces<E>(t, 2 * hf + 1);
                pf[2] = get_pieces<E>(t, 5 - hf);
            }
        };
        if constexpr (MODE == FORWARD) {
            const Keys at;
            E *const op = o + b * a.o.batch + h * a.o.head + col0 + 16 * w;
            const int there = a.Dv - (col0 + 16 * w + 4 * gr);
            v4f y[2], old[2];
            auto finish = [&](int i) {                // O of chunk i, of which `old` is exp(G) Q S
                const v4f *const uc = xu[i & 1] + w * XU + lane;
                const v4f was[2] = {old[0], old[1]};
                auto add = [&](const Pieces<E> &u0, const Pieces<E> &u1) {
#pragma unroll
                    for (int n = NP - 1; n >= 0; --n)
#pragma unroll
                        for (int m = 0; m <= n; ++m) {
                            old[0] = Mx<E>::mma(old[0], u0.p[n - m], pf[0].p[m]);
                            old[1] = Mx<E>::mma(old[1], u0.p[n - m], pf[1].p[m]);
                            old[1] = Mx<E>::mma(old[1], u1.p[n - m], pf[2].p[m]);
                        }
                };
                add(split<E>(uc[0], uc[kWave]), split<E>(uc[2 * kWave], uc[3 * kWave]));
                const float all_of = (old[1][0] + old[1][1]) + (old[1][2] + old[1][3]);
                if (__builtin_expect(__any(all_of != all_of), 0)) {
                    // The same with U, whose rows that are not finite have reached all tokens, times zeros of P
                    v4f x[4];
                    int first = kChunk;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        x[t] = uc[t * kWave];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(__builtin_fabsf(x[t][e]) < kLimit<E>)) first = first < 16 * t + 4 * gr + e ? first : 16 * t + 4 * gr + e;
                    }
                    first = least_of_columns(first);
                    keep_before(x, first, 0.0f);
                    old[0] = was[0], old[1] = was[1];
                    add(split<E>(x[0], x[1]), split<E>(x[2], x[3]));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int from = __shfl(first, 4 * gr + e);
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            if (16 * tile[t] + l >= from) old[t][e] = __builtin_nanf("");
                    }
                }
                const int64_t left = a.T - (int64_t)i * kChunk, real = len - (int64_t)i * kChunk;
                E *const oc = op + (int64_t)i * kChunk * a.o.token;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    typename Vec<E>::v4 out;
                    const int token = 16 * tile[t] + l;
#pragma unroll
                    for (int e = 0; e < 4; ++e) out[e] = token < real ? (E)(scale * old[t][e]) : (E)0.0f;      // (a row of zeros times a state that is not finite is not zero)
                    if constexpr (FULL) {             // rows behind the last token lie behind the end of the buffer
                        const int st = (int)a.o.token * 2, many = left < kChunk ? (int)left : kChunk;
                        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, out), rsrc(oc, (unsigned)((many - 1) * st + 32)), token * st + 8 * gr, 0, 0);
                    } else if (token < left) {
                        E *const to = oc + token * a.o.token + 4 * gr;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < there) to[e] = out[e];
                    }
                }
            };
            barrier();
            for (int i = 0; i < chunks; ++i) {
                const int p = i & 1;
                const E *const sc = (const E *)(xs[0] + w * XS), *const qc = qs[p];
                Frag<E> qf[KB][2];
                Pieces<E> sf[KB];
                float gm[2];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    sf[kb] = get_pieces<E>(sc, kb);
#pragma unroll
                    for (int t = 0; t < 2; ++t) qf[kb][t] = at.rows(qc, tile[t], kb);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    y[t] = zero;
                    gm[t] = fs[p][16 * tile[t] + l];
                }
                barrier();                            // (the reads are out: the states' wavefronts do not wait for the products)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int n = NP - 1; n >= 0; --n)
#pragma unroll
                        for (int t = 0; t < 2; ++t) y[t] = Mx<E>::mma(y[t], sf[kb].p[n], qf[kb][t]);
                if (i > 0) finish(i - 1);
                fetch(i);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) old[t][e] = gm[t] * y[t][e];
                barrier();
            }
            if (chunks > 0) finish(chunks - 1);
        } else {
            // chunk i's terms with dO; exp(G) of the chunk straight from memory
            auto terms = [&](int i) {
                const int p = i & 1;
                const E *const vc = vs[p], *const qc = qs[p];
                const float *const gp = ws.factors + (head * ws.chunks + first + i * step) * (int64_t)(3 * kChunk);
                v4f *const zc = xu[p] + w * XU + lane, *const yc = xs[p] + w * XS + HT * hf * kWave + lane;
                v4f g4[4], y[4], z[2];
#pragma unroll
                for (int t = 0; t < 4; ++t) g4[t] = *(const v4f *)(gp + 16 * t + 4 * gr);
                const Frag<E> o0 = Tile<E, W>::cols_of(vc, 0, w), o1 = Tile<E, W>::cols_of(vc, 1, w);
                Frag<E> cf[HT][2];
#pragma unroll
                for (int j = 0; j < HT; ++j) {
                    cf[j][0] = cols(qc, 0, j);
                    cf[j][1] = cols(qc, 1, j);
                }
                __builtin_amdgcn_sched_barrier(0);
                z[0] = z[1] = zero;
#pragma unroll
                for (int n = NP - 1; n >= 0; --n) {
                    z[0] = Mx<E>::mma(z[0], pf[0].p[n], o0);
                    z[1] = Mx<E>::mma(z[1], pf[2].p[n], o1);
                    z[0] = Mx<E>::mma(z[0], pf[1].p[n], o1);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t)           // dO in accumulator layout is its operand
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[t][e] = scale * g4[t][e] * (float)(t < 2 ? o0 : o1)[4 * (t & 1) + e];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[t][e] *= scale;
                    zc[tile[t] * kWave] = z[t];
                }
                const Pieces<E> y0 = split<E>(y[0], y[1]), y1 = split<E>(y[2], y[3]);
                v4f r[HT];
#pragma unroll
                for (int j = 0; j < HT; ++j) r[j] = zero;
#pragma unroll
                for (int n = NP - 1; n >= 0; --n) {
#pragma unroll
                    for (int j = 0; j < HT; ++j) r[j] = Mx<E>::mma(r[j], cf[j][0], y0.p[n]);
#pragma unroll
                    for (int j = 0; j < HT; ++j) r[j] = Mx<E>::mma(r[j], cf[j][1], y1.p[n]);
                }
#pragma unroll
                for (int j = 0; j < HT; ++j) yc[j * kWave] = r[j];
            };
            if (chunks > 0) fetch(0);
            barrier();
            if (chunks > 0) {
                terms(0);
                if (chunks > 1) fetch(1);
            }
            barrier();
            for (int i = 0; i < chunks; ++i) {
                barrier();
                if (i + 1 < chunks) {
                    terms(i + 1);
                    if (i + 2 < chunks) fetch(i + 2);
                }
                barrier();
            }
        }
        return;
    }

    // Those that load.  Of the i-th chunk, K and (forward) Q and V are staged during the chunk before; backward Q and dO one earlier; T as its chunk begins,
    // when the one before has been read.  Loads go out a chunk before they are staged, whether there is such a chunk or not (the last one again):
    // what is waited for is then the same number of loads every time, and none of the later ones.
    auto there = [&](int i) { return i < chunks ? i : chunks - 1; };
    const int tid = threadIdx.x - (scan_threads(NS, MODE) - 2 * NL);
    const E *const kp = k + b * a.k.batch + hk * a.k.head, *const qp = q + b * a.q.batch + hk * a.q.head;
    const E *const vp = MODE == BACKWARD ? o + b * a.o.batch + h * a.o.head + col0 : v + b * a.v.batch + h * a.v.head + col0;
    const int64_t vstep = MODE == BACKWARD ? a.o.token : a.v.token;
    auto tokens_at = [&](int i, int64_t &t0) {
        t0 = (int64_t)(first + there(i) * step) * kChunk;
        return len - t0 < kChunk ? (int)(len - t0) : kChunk;
    };
    if (tid >= NL) {                                  // T, the factors and Q
        constexpr int TN = TRI / 16 / NL;
        static_assert(TN * 16 * NL == TRI, "");
        const int t = tid - NL;
        v4u tr[TN];
        unsigned fr[2];
        Rows<E, DK, NL, FULL> qr;
        auto fetch_q = [&](int i) {
            int64_t t0;
            const int n = tokens_at(i, t0);
            if (QUERIES) qr.load(qp + t0 * a.q.token, a.q.token, n, a.Dk, t);
        };
        auto stage_q = [&](int p) {
            if (QUERIES) qr.store(qs[p], t);
        };
        auto fetch_tri = [&](int i) {
            const v4u *const tp = (const v4u *)tri_of(there(i), T_AT) + t;
#pragma unroll
            for (int j = 0; j < TN; ++j) tr[j] = tp[j * NL];
        };
        auto fetch_factors = [&](int i) {             // (nothing behind the 192)
            const __amdgpu_buffer_rsrc_t from = rsrc(ws.factors + (head * ws.chunks + first + there(i) * step) * (int64_t)(3 * kChunk), 3 * kChunk * 4);
            fr[0] = __builtin_amdgcn_raw_buffer_load_b32(from, 4 * t, 0, 0);
            fr[1] = __builtin_amdgcn_raw_buffer_load_b32(from, 4 * (t + NL), 0, 0);
        };
        auto stage_tri = [&]() {
#pragma unroll
            for (int j = 0; j < TN; ++j) m.ts[t + j * NL] = tr[j];
        };
        auto stage_factors = [&](int p) {
            fs[p][t] = __uint_as_float(fr[0]);
            fs[p][t + NL] = __uint_as_float(fr[1]);
        };
        if (chunks > 0) {
            fetch_tri(0);
            fetch_factors(0);
            fetch_q(0);
            stage_tri();
            stage_factors(0);
            stage_q(0);
            fetch_tri(1);
            fetch_factors(1);
            fetch_q(1);
        }
        barrier();
        if constexpr (MODE == BACKWARD) {
            if (chunks > 0) {
                stage_q(1);
                fetch_q(2);
            }
            barrier();
        }
        for (int i = 0; i < chunks; ++i) {
            if (i > 0) {
                stage_tri();
                fetch_tri(i + 1);
            }
            barrier();
            stage_factors((i + 1) & 1);
            fetch_factors(i + 2);
            stage_q(MODE == BACKWARD ? i & 1 : (i + 1) & 1);
            fetch_q(MODE == BACKWARD ? i + 3 : i + 2);
            barrier();
        }
        return;
    }
    Rows<E, DK, NL, FULL> kr;                         // K, and V or dO
    Rows<E, W, NL, FULL> vr;
    auto fetch_keys = [&](int i) {
        int64_t t0;
        const int n = tokens_at(i, t0);
        kr.load(kp + t0 * a.k.token, a.k.token, n, a.Dk, tid);
    };
    auto fetch_rest = [&](int i) {
        int64_t t0;
        const int n = tokens_at(i, t0);
        vr.load(vp + t0 * vstep, vstep, n, a.Dv - col0, tid);
    };
    auto stage_keys = [&](int p) { kr.store(ks[p], tid); };
    auto stage_rest = [&](int p) { vr.store(vs[p], tid); };

    if (chunks > 0) {
        fetch_keys(0);
        fetch_rest(0);
        stage_keys(0);
        stage_rest(0);
        fetch_keys(1);
        fetch_rest(1);
    }
    barrier();
    if constexpr (MODE == BACKWARD) {
        if (chunks > 0) {
            stage_rest(1);
            fetch_rest(2);
        }
        barrier();
    }
    for (int i = 0; i < chunks; ++i) {
        barrier();
        stage_keys((i + 1) & 1);
        fetch_keys(i + 2);
        if constexpr (MODE != BACKWARD) {
            stage_rest((i + 1) & 1);
            fetch_rest(i + 2);
        } else {
            stage_rest(i & 1);
            fetch_rest(i + 3);
        }
        barrier();
    }
    if constexpr (MODE == FORWARD) {                  // whole chunks of tokens that are not there
        const int width = a.Dv - col0 < W ? a.Dv - col0 : W;
        E *const zp = o + b * a.o.batch + h * a.o.head + col0;
        for (int64_t t = (int64_t)chunks * kChunk + tid / W; t < a.T; t += NL / W)
            if (tid % W < width) zp[t * a.o.token + tid % W] = (E)0.0f;
    }
}

template <class E, int MODE>
hipError_t launch(const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws, const DeltaArgs &a, hipStream_t s)
{
    const int64_t heads = a.B * a.Hv;
    // the gradients read whole blocks of 32 columns of what is kept
    const int cols = MODE == FORWARD ? a.Dv : ws.cols;
    auto go = [&](auto dk, auto ns) {
        constexpr int DK = decltype(dk)::value, NS = decltype(ns)::value, W = 16 * NS;
        // (every block of columns that the grid has must be one of the values: whole loads do not stop at the end of a head)
        const bool full = a.Dk == DK && a.Dv == cols && cols % W == 0 && full_rows<E>(a.q, DK, q) && full_rows<E>(a.k, DK, k) && full_rows<E>(a.v, W, v) &&
                          full_rows<E>(a.o, W, o);
        auto *kernel = full ? delta_scan_kernel<E, DK, NS, MODE, true> : delta_scan_kernel<E, DK, NS, MODE, false>;
        static std::atomic<uint64_t> raised[2] = {{0}, {0}};
        constexpr int bytes = sizeof(ScanLds<E, DK, NS, MODE>);
        if (const hipError_t e = raise_lds((const void *)kernel, bytes, raised[full])) return e;
        dim3 grid;
        if (!spread(heads, scan_threads(NS, MODE), grid, (unsigned)((cols + W - 1) / W))) return kNotTaken;
        hipLaunchKernelGGL(kernel, grid, dim3(scan_threads(NS, MODE)), bytes, s, (const E *)q, (const E *)k, (const E *)v,
                           (E *)o, state, ws, a);
        return hipGetLastError();
    };
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I64 = std::integral_constant<int, 64>;
    using I128 = std::integral_constant<int, 128>;
    const bool pairs = heads * ((cols + 31) / 32) >= device_cus();
    if (a.Dk <= 64) return pairs ? go(I64(), I2()) : go(I64(), I1());
    return pairs ? go(I128(), I2()) : go(I128(), I1());
}

}  // namespace

hipError_t launch_delta_scan_16(int dtype, int mode, const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws,
                                const DeltaArgs &a, hipStream_t s)
{
    auto by_mode = [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        if (mode == FORWARD) return launch<E, FORWARD>(q, k, v, o, state, ws, a, s);
        if (mode == KEEP) return launch<E, KEEP>(q, k, v, o, state, ws, a, s);
        return launch<E, BACKWARD>(q, k, v, o, state, ws, a, s);
    };
    return dtype == SWS_DTYPE_BF16 ? by_mode((__bf16 *)nullptr) : by_mode((_Float16 *)nullptr);
}

}  // namespace sws

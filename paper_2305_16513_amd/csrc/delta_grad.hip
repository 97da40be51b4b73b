// The last pass of the gated delta rule's gradients, for all chunks side by side: from what the passes from chunk to chunk have left (U, dR, the
// states S before the chunks and the gradients dS of those behind them) the gradients of q, k, v, g and beta.
//
//   dP_ij = scale D_ij dO_i.U_j (j <= i),   M_ij = -beta_i D_ij dR_i.U_j (j < i)
//   dq = dP K + scale exp(G) (dO S^T)
//   dk = M K - beta exp(G) (dR S^T)                       (k in its own row: "row")
//      + M^T K + dP^T Q + exp(G_63 - G) (U dS^T)          (k in later rows: "column")
//   dv = beta dR,   dbeta_i = dR_i.V_i - exp(G_i) k_i.(dR S^T)_i - sum_j D_ij (dR_i.U_j) (k_i.k_j)
//   dG_i = q_i.dq_i + k_i.dk_i(row) - k_i.dk_i(column),   dG_63 += exp(G_63) <S, dS> + sum_j k_j.(exp(G_63 - G) U dS^T)_j
//   dg_i = sum of dG_j, j >= i
// (G_i enters as exp(G_i) with q_i and with k_i in its own row, as exp(-G_i) with k_i in later rows.)
//
// A workgroup takes a chunk of one key head and, one after the other, the value heads that read it, whose dq and dk it adds in registers: no
// atomics.  Four of its eight wavefronts take dP and what dq and dk have of it, of S and of dS; the others M and what dk has of it and of S.  Each owns 32 tokens x
// half of the keys' elements of the products with the states, so that an operand of those is read from LDS for two tiles of tokens, and the
// blocks of dP or M that one tile of 16 tokens is in: as rows and as columns, so that they become the next products' operands, which go
// from wavefront to wavefront through LDS.  The products over the values' elements are taken 32 of them at a time.
// Bound by HBM, of whose bytes the states and their gradients, Dk Dv numbers of 32 bits each per chunk, are most, while columns are taken, and by one workgroup a CU (118 KB of LDS, all registers of two
// wavefronts a SIMD) before them and behind them, when nothing is loaded; the next 32 columns of everything are on their way to registers during the products of these, and
// are cut into pieces on the way from there to LDS.
// bf16, 4096 chunks and states of 128 x 128: 493 us (shortest 456) for 1.33 GB, which a copy takes 259 for.  Counters: vector units 42 % of the time, matrix units 21 %, LDS 44 %.
// (With fp32 sums kept over heads that share keys, some 50 registers go to scratch between the columns' loops, none within.)
#include "delta.h"

namespace sws {

namespace {

constexpr int kThreads = 512;

struct GradWs {
    const void *u, *r, *s, *ds;                       // U, dR, S, dS as the passes before have left them (see Kept)
    const float *scales;                              // fp16: of U and S, and of dR and dS
    int chunks, cols;
};

template <class E>
__device__ __forceinline__ float whole(const Pieces<E> &x, int e)
{
    float f = 0;
#pragma unroll
    for (int n = Mx<E>::NP - 1; n >= 0; --n) f += (float)x.p[n][e];
    return f;
}

template <class E, class G, int DK, bool MANY, bool FULL>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void delta_grad_kernel(const E *__restrict__ q, const E *__restrict__ k, const E *__restrict__ v, const G *__restrict__ g, const G *__restrict__ beta,
                       const E *__restrict__ go, E *__restrict__ gq, E *__restrict__ gk, E *__restrict__ gv, G *__restrict__ gg,
                       G *__restrict__ gbeta, GradWs ws, DeltaArgs a, Steps sq, Steps sk, Steps sv)
{
    constexpr int NP = Mx<E>::NP, KB = DK / 32, KH = DK / 32;    // a wavefront's tiles of 16 of the keys' elements
    typedef Tile<E, DK> Keys;                         // of 64 tokens
    typedef Tile<E, 32> Values;                       // of 64 tokens, 32 of their values' elements
    constexpr int SG = KB * Kept<E>::OPERAND, UG = 2 * Kept<E>::OPERAND;         // bytes of 16 columns in LDS
    struct Block {                                    // of 32 columns of the state S, dS, U, dR as operands, dO and V
        char s[2 * SG], d[2 * SG], u[2 * UG], r[2 * UG];
        E o[Values::size(kChunk)], v[Values::size(kChunk)];
    };
    // After the columns dP and M as operands, then dq and dk; in the place of K and Q what dk has of dP and dS
    constexpr int BYTES = (int)sizeof(Block), AFTER = 8 * 3 * kWave * (int)sizeof(Pieces<E>), OUT = 2 * (int)sizeof(E) * Keys::size(kChunk);
    constexpr int MOST = BYTES > AFTER ? (BYTES > OUT ? BYTES : OUT) : (AFTER > OUT ? AFTER : OUT);
    __shared__ __align__(16) char lds[MOST];
    __shared__ __align__(16) E keys[2][Keys::size(kChunk)];
    static_assert(sizeof(float) * kChunk * DK <= sizeof keys, "");
    __shared__ double sums[kChunk];
    __shared__ float betas[kChunk], dbs[kChunk], dots[2][2][kChunk], xdots[2][2][kChunk], parts[8];
    Block &m4 = *(Block *)lds;
    E *const ks = keys[0], *const qs = keys[1], *const outq = (E *)lds, *const outk = outq + Keys::size(kChunk);
    E *const operands = (E *)lds;
    v4f *const ex = (v4f *)keys;
    int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave), w = wave % 4, l = tid % 16, gr = tid % kWave / 16;
    const int th = w / 2, dh = w & 1;                 // tiles 2 th, 2 th + 1 of the tokens, KH dh ... of the keys' elements; w's own tile of tokens is 2 th + dh
    const bool second = wave >= 4;                    // M's wavefronts
    const int64_t unit = group_of() / (unsigned)ws.chunks, b = (unsigned)unit / (unsigned)a.Hk;
    const int c = group_of() % (unsigned)ws.chunks;
    if (b >= a.B) return;
    const int hk = (int)(unit - b * a.Hk), share = a.Hv / a.Hk;
    const int64_t t0 = (int64_t)c * kChunk, left = tokens_of(a, b) - t0;
    const int n = left <= 0 ? 0 : left < kChunk ? (int)left : kChunk;
    const int rows = a.T - t0 < kChunk ? (int)(a.T - t0) : kChunk;       // tokens of the chunk that have gradients, if only zeros
    const v4f zero = {0, 0, 0, 0};

    v4f total[MANY ? 2 : 1][MANY ? KH : 1];           // of several heads: dq, or dk
    if constexpr (MANY)
#pragma unroll
        for (int i = 0; i < KH; ++i) total[0][i] = total[1][i] = zero;
    // An element of a key or query per lane, four tokens: to the rows that go out at the end
    auto to_row = [&](E *out, int tt, int i, v4f x) {
        const int d = 16 * (KH * dh + i) + l;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[Keys::at(16 * (2 * th + tt) + 4 * gr + e, d / 4) + d % 4] = (E)x[e];
    };
    auto rows_out = [&]() {
        constexpr int PER = 16 / (int)sizeof(E), UNITS = DK / PER;
        E *const qp = gq + b * sq.batch + t0 * sq.token + hk * sq.head, *const kp = gk + b * sk.batch + t0 * sk.token + hk * sk.head;
        for (int u = tid; u < rows * UNITS; u += kThreads) {
            const int r = u / UNITS, c0 = u % UNITS * PER, from = Keys::at(r, c0 / 4);
            const bool real = r < n;                  // (others are zeros, also where what they were multiplied with is not finite)
            const v4u none = {0, 0, 0, 0}, x = real ? *(const v4u *)(outq + from) : none, y = real ? *(const v4u *)(outk + from) : none;
            if constexpr (FULL) {
                *(v4u *)(qp + r * sq.token + c0) = x;
                *(v4u *)(kp + r * sk.token + c0) = y;
            } else
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    if (c0 + e < a.Dk) {
                        qp[r * sq.token + c0 + e] = real ? outq[from + e] : (E)0.0f;
                        kp[r * sk.token + c0 + e] = real ? outk[from + e] : (E)0.0f;
                    }
        }
    };

    for (int hs = 0; hs < (MANY ? share : 1); ++hs) {
        const int h = hk * share + hs;
        int lane, l, gr, mine;                        // mine: token of the wavefront's own tile
        Keys ak(tid);
        // Not known to be what they were before: addresses are not kept in registers until they are needed.  (With more of them than registers, the compiler has copied one where the lanes
        // of rows that are not there were switched off, behind the loads of the others, and left theirs behind.)
        auto whereabouts = [&]() {
            asm volatile("" : "+v"(tid));
            lane = tid % kWave, l = tid % 16, gr = lane / 16, mine = 16 * w + l;
            ak = Keys(tid);
        };
        whereabouts();
        const Values av(tid);
        const int64_t at = ((b * a.Hv + h) * ws.chunks + c);
        G *const ggp = gg + (b * a.T + t0) * a.Hv + h, *const gbp = gbeta + (b * a.T + t0) * a.Hv + h;
        if (n == 0) {                                 // (the whole workgroup)
            for (int i = tid; i < rows * a.Dv; i += kThreads) gv[b * sv.batch + (t0 + i / a.Dv) * sv.token + h * sv.head + i % a.Dv] = (E)0.0f;
            if (tid < rows) ggp[(int64_t)tid * a.Hv] = gbp[(int64_t)tid * a.Hv] = (G)0.0f;
            continue;
        }
        // What is made of U or S and of dR or dS has both scales, and so has what dO is multiplied into, by way of `scale`
        const float rise = kScaled<E> ? ws.scales[2 * (b * a.Hv + h)] : 1.0f, grise = kScaled<E> ? ws.scales[2 * (b * a.Hv + h) + 1] : 1.0f;
        const float fall = 1.0f / rise, gfall = 1.0f / grise, scale = kScaled<E> ? a.scale * grise : a.scale;
        auto whole_again = [&](float f) { return kScaled<E> ? f * fall * gfall : f; };
        const int64_t kept = at * (ws.cols / 16);
        const char *const up = (const char *)ws.u + kept * Kept<E>::rows(), *const rp = (const char *)ws.r + kept * Kept<E>::rows();
        const char *const sp = (const char *)ws.s + kept * Kept<E>::state(DK), *const dp = (const char *)ws.ds + kept * Kept<E>::state(DK);
        const E *const op = go + b * a.o.batch + t0 * a.o.token + h * a.o.head, *const vp = v + b * a.v.batch + t0 * a.v.token + h * a.v.head;
        float inner = 0;                              // <S, dS>
        // The next 32 columns are on their way to registers during the products of these.  S and dS have 64 KB lanes' shares of operands, U and dR 256 together: a thread
        // takes one of S, the same of dS and one of U or dR; with KB = 2 half of the threads S and dS, the others U and dR.  Eight threads a row of dO and V.
        typedef typename Vec<E>::v4 V4;
        V4 ov, vv;
        v4f s4[2], d4[2], u4[2];
        const bool low = wave < 4;
        auto fetch = [&](int d0) {
            const int64_t so = (int64_t)d0 / 16 * Kept<E>::state(DK), uo = (int64_t)d0 / 16 * Kept<E>::rows();
            if constexpr (KB == 4) {
                Kept<E>::load(sp + so + 2048 * wave, lane, s4);
                Kept<E>::load(dp + so + 2048 * wave, lane, d4);
                Kept<E>::load((low ? up : rp) + uo + 2048 * w, lane, u4);
            } else {
                Kept<E>::load((low ? sp + so : up + uo) + 2048 * w, lane, s4);
                Kept<E>::load((low ? dp + so : rp + uo) + 2048 * w, lane, d4);
            }
            const int r = tid / 8, c4 = 4 * (tid % 8);
            if constexpr (FULL) {                     // rows that are not there lie behind the end of a buffer
                constexpr int SIZE = (int)sizeof(E);
                auto row = [&](const E *from, const Steps &s) {
                    const __amdgpu_buffer_rsrc_t b = rsrc(from + d0, (unsigned)((n - 1) * (int)s.token * SIZE + 32 * SIZE));
                    const int off = r < n ? r * (int)s.token * SIZE + c4 * SIZE : 0x7ffffff0;
                    if constexpr (SIZE == 4) return __builtin_bit_cast(V4, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0));
                    else return __builtin_bit_cast(V4, __builtin_amdgcn_raw_buffer_load_b64(b, off, 0, 0));
                };
                ov = row(op, a.o);
                vv = row(vp, a.v);
            } else {
                ov = vv = V4{};
                if (r < n) {
                    const E *po = op + r * a.o.token + d0 + c4, *pv = vp + r * a.v.token + d0 + c4;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < a.Dv - d0 - c4) {
                            ov[e] = po[e];
                            vv[e] = pv[e];
                        }
                }
            }
        };
        auto stage = [&](int d0) {
            __syncthreads();                          // the last columns have been read
            if constexpr (KB == 4) {
                Kept<E>::lay(m4.s, wave, lane, s4);
                Kept<E>::lay(m4.d, wave, lane, d4);
                Kept<E>::lay(low ? m4.u : m4.r, w, lane, u4);
            } else {
                Kept<E>::lay(low ? m4.s : m4.u, w, lane, s4);
                Kept<E>::lay(low ? m4.d : m4.r, w, lane, d4);
            }
            *(V4 *)(m4.o + Values::at(tid / 8, tid % 8)) = ov;
            *(V4 *)(m4.v + Values::at(tid / 8, tid % 8)) = vv;
            if (KB == 4 || low)
#pragma unroll
                for (int e = 0; e < 4; ++e) inner += s4[0][e] * d4[0][e] + s4[1][e] * d4[1][e];
            __syncthreads();
            if (d0 + 32 < ws.cols) fetch(d0 + 32);
        };
        // The five blocks of dP or M that the wavefront's own tile of tokens is in: x[t], t <= w, rows are tokens j of tile t, columns tokens i of its own;
        // x[t + 1], t >= w, rows are tokens i of tile t, columns tokens j of its own.  (Slots, not tiles: which ones there are depends on
        // the wavefront, and an accumulator under a condition is two.)
        v4f x[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) x[i] = zero;
        // the block in every slot times its decay, as f(i, j, value, t or -1, e) makes it, left as operands: of a contraction over j the first 32, 0, over i
        // the last 32, 2, and of those that are left the one that has more than zeros, 1
        auto leave = [&](auto &&f) {
            const double gm = sums[mine];
            v4f m[8];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                m[t] = m[4 + t] = zero;
                if (t <= w) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = 16 * t + 4 * gr + e;
                        m[t][e] = f(mine, j, j <= mine ? x[t][e] * decay<E>((float)(gm - sums[j])) : 0.0f, t, e);
                    }
                }
                if (t >= w) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 16 * t + 4 * gr + e;
                        m[4 + t][e] = f(i, mine, i >= mine ? x[t + 1][e] * decay<E>((float)(sums[i] - gm)) : 0.0f, -1, e);
                    }
                }
            }
            __syncthreads();                          // the blocks have been read
            put_pieces<E>(operands, wave * 3, split<E>(m[0], m[1]), tid);
            put_pieces<E>(operands, wave * 3 + 1, th ? split<E>(m[2], m[3]) : split<E>(m[4], m[5]), tid);
            put_pieces<E>(operands, wave * 3 + 2, split<E>(m[6], m[7]), tid);
            __syncthreads();
        };
        // operand i of tile 2 th + tt
        auto operand = [&](int tt, int i) { return get_pieces<E>(operands, (4 * second + 2 * th + tt) * 3 + i, tid); };
        float dot[2][4] = {}, xdot[2][4] = {};        // of rows of the tiles, with q and k
        auto leave_dots = [&]() {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d = sum16(dot[tt][e]), y = sum16(xdot[tt][e]);
                    if (l == 0) {
                        dots[second][dh][16 * (2 * th + tt) + 4 * gr + e] = d;
                        xdots[second][dh][16 * (2 * th + tt) + 4 * gr + e] = y;
                    }
                }
        };

        if (hs) __syncthreads();                      // the last head's rows and sums have been read
        {
            Rows<E, DK, kThreads, FULL> kr, qr;
            kr.load(k + b * a.k.batch + t0 * a.k.token + hk * a.k.head, a.k.token, n, a.Dk, tid);
            qr.load(q + b * a.q.batch + t0 * a.q.token + hk * a.q.head, a.q.token, n, a.Dk, tid);
            double s = 0;
            float bt = 0;
            if (wave == 0 && lane < n) {
                s = (double)gate((float)g[b * a.g.batch + (t0 + lane) * a.g.token + h * a.g.head]);
                bt = (float)beta[b * a.beta.batch + (t0 + lane) * a.beta.token + h * a.beta.head];
            }
            fetch(0);
            kr.store(ks, tid);
            qr.store(qs, tid);
            if (wave == 0) {
#pragma unroll
                for (int d = 1; d < kWave; d <<= 1) {
                    const double t = __shfl_up(s, d);
                    if (lane >= d) s += t;
                }
                sums[lane] = s;
                betas[lane] = bt;
            }
        }
        if (!second) {
            v4f x1[2][KH], x3[2][KH];                 // dO S^T, U dS^T
#pragma unroll
            for (int i = 0; i < KH; ++i) x1[0][i] = x1[1][i] = x3[0][i] = x3[1][i] = zero;
#pragma unroll 1
            for (int d0 = 0; d0 < ws.cols; d0 += 32) {
                stage(d0);
                const Frag<E> om[2] = {av.rows(m4.o, 2 * th, 0), av.rows(m4.o, 2 * th + 1, 0)};
                Pieces<E> um[2];
                Kept<E>::both(m4.u, UG, th, um, tid);
#pragma unroll
                for (int i = 0; i < KH / 2; ++i) {
                    Pieces<E> st[2];
                    Kept<E>::both(m4.s, SG, KH / 2 * dh + i, st, tid);
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int m = 0; m < 2; ++m) x1[tt][2 * i + m] = mma<E>(x1[tt][2 * i + m], om[tt], st[m]);
                    __builtin_amdgcn_sched_barrier(0);    // (or all the reads go out first, into more registers than there are)
                    Kept<E>::both(m4.d, SG, KH / 2 * dh + i, st, tid);
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int m = 0; m < 2; ++m) x3[tt][2 * i + m] = mma<E>(x3[tt][2 * i + m], um[tt], st[m]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                const Frag<E> o1 = dh ? om[1] : om[0];
                const Pieces<E> u1 = dh ? um[1] : um[0];
#pragma unroll
                for (int t = 0; t < 5; ++t) {
                    Pieces<E> l4, r4;                 // left and right
                    if (t <= w) {
                        l4 = Kept<E>::columns(m4.u, UG, t, tid);
#pragma unroll
                        for (int m = 0; m < NP; ++m) r4.p[m] = o1;
                    } else {
                        const Frag<E> ot = av.rows(m4.o, t - 1, 0);
#pragma unroll
                        for (int m = 0; m < NP; ++m) l4.p[m] = ot;
                        r4 = u1;
                    }
#pragma unroll
                    for (int m = NP - 1; m >= 0; --m) x[t] = Mx<E>::mma(x[t], l4.p[m], r4.p[m]);
                }
            }
            whereabouts();
            inner = sum_lanes(inner, kWave);
            if (lane == 0) parts[wave] = inner;
            leave([&](int, int, float y, int, int) { return scale * y; });
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const Pieces<E> p0 = operand(tt, 0), p1 = operand(tt, 1), p3 = operand(tt, 2);
                float ga[4], de[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double g1 = sums[16 * (2 * th + tt) + 4 * gr + e];
                    ga[e] = scale * decay<E>((float)g1);
                    de[e] = decay<E>((float)(sums[kChunk - 1] - g1));
                }
#pragma unroll
                for (int i = 0; i < KH; ++i) {
                    const int j = KH * dh + i;
                    const v4f kv = widen(ak.column_of(ks, 2 * th + tt, j, tid)), qv = widen(ak.column_of(qs, 2 * th + tt, j, tid));
                    v4f y1 = x1[tt][i], y3 = x3[tt][i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y1[e] *= ga[e];
                        y3[e] *= de[e];
                        xdot[tt][e] += kv[e] * y3[e];
                    }
                    y1 = mma<E>(y1, p0, ak.cols_of(ks, 0, j, tid));
                    if (th) y1 = mma<E>(y1, p1, ak.cols_of(ks, 1, j, tid));       // (the upper blocks are zeros)
                    else y3 = mma<E>(y3, p1, ak.cols_of(qs, 0, j, tid));
                    y3 = mma<E>(y3, p3, ak.cols_of(qs, 1, j, tid));
#pragma unroll
                    for (int e = 0; e < 4; ++e) dot[tt][e] += qv[e] * y1[e] - kv[e] * y3[e];
                    x1[tt][i] = y1;
                    x3[tt][i] = y3;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            leave_dots();
            __syncthreads();                          // K, Q and the operands have been read
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < KH; ++i) {
                    ex[((w * 2 + tt) * KH + i) * kWave + lane] = x3[tt][i];
                    if constexpr (kScaled<E>)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x1[tt][i][e] = whole_again(x1[tt][i][e]);
                    if constexpr (MANY) total[tt][i] += x1[tt][i];
                    else to_row(outq, tt, i, x1[tt][i]);
                }
            if (wave == 0) {
                float s = (dots[0][0][lane] + dots[0][1][lane]) + (dots[1][0][lane] + dots[1][1][lane]);
                const float all = sum_lanes(xdots[0][0][lane] + xdots[0][1][lane], kWave);
                if (lane == kChunk - 1)
                    s += decay<E>((float)sums[kChunk - 1]) * (((parts[0] + parts[1]) + (parts[2] + parts[3])) + ((parts[4] + parts[5]) + (parts[6] + parts[7]))) + all;
#pragma unroll
                for (int d = 1; d < kWave; d <<= 1) {
                    const float t = __shfl_down(s, d);
                    if (lane + d < kWave) s += t;
                }
                if (lane < rows) ggp[(int64_t)lane * a.Hv] = (G)(lane < n ? whole_again(s) : 0.0f);
            }
            __syncthreads();
        } else {
            v4f x2[2][KH], vd = zero;                 // dR S^T; dR V^T of the own tile: its diagonal is dR.V
#pragma unroll
            for (int i = 0; i < KH; ++i) x2[0][i] = x2[1][i] = zero;
            E *const gvp = gv + b * sv.batch + t0 * sv.token + h * sv.head + mine * sv.token + 4 * gr;
#pragma unroll 1
            for (int d0 = 0; d0 < ws.cols; d0 += 32) {
                stage(d0);
                Pieces<E> rm[2], um;
                Kept<E>::both(m4.r, UG, th, rm, tid);
#pragma unroll
                for (int i = 0; i < KH / 2; ++i) {
                    Pieces<E> st[2];
                    Kept<E>::both(m4.s, SG, KH / 2 * dh + i, st, tid);
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                        for (int m = 0; m < 2; ++m) x2[tt][2 * i + m] = mma<E>(x2[tt][2 * i + m], rm[tt], st[m]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                const Pieces<E> r1 = dh ? rm[1] : rm[0];
                um = Kept<E>::columns(m4.u, UG, w, tid);
                vd = mma<E>(vd, r1, av.rows(m4.v, w, 0));
                if (mine < rows) {                    // dv: elements 4 gr .. and 16 + 4 gr .. of the block
                    const float bt = betas[mine];
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        typename Vec<E>::v4 out;
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[e] = mine < n ? (E)((kScaled<E> ? gfall * bt : bt) * whole<E>(r1, 4 * m + e)) : (E)0.0f;
                        if constexpr (FULL) *(typename Vec<E>::v4 *)(gvp + d0 + 16 * m) = out;
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (d0 + 16 * m + 4 * gr + e < a.Dv) gvp[d0 + 16 * m + e] = out[e];
                    }
                }
#pragma unroll
                for (int t = 0; t < 5; ++t) {
                    const Pieces<E> l4 = Kept<E>::columns(t <= w ? m4.u : m4.r, UG, t <= w ? t : t - 1, tid), r4 = t <= w ? r1 : um;
                    x[t] = mma<E>(x[t], l4, r4);
                }
            }
            whereabouts();
            inner = sum_lanes(inner, kWave);
            if (lane == 0) parts[wave] = inner;
            float db = 0;                             // of token `mine`, the part of this lane's rows
            v4f kk = zero;
            leave([&](int i, int j, float y, int t, int e) {
                if (t >= 0 && e == 0) {               // (t, e in order)
                    kk = zero;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) kk = Mx<E>::mma(kk, ak.rows(ks, t, kb), ak.rows(ks, w, kb));
                }
                const float m = i > j ? -y : 0.0f;
                if (t >= 0) db += m * kk[e];
                return betas[i] * m;
            });
            db += __shfl_xor(db, 16);
            db += __shfl_xor(db, 32);
            if (gr == 0) dbs[mine] = db;
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const Pieces<E> p0 = operand(tt, 0), p1 = operand(tt, 1), p3 = operand(tt, 2);
                float ga[4], be[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    be[e] = betas[16 * (2 * th + tt) + 4 * gr + e];
                    ga[e] = decay<E>((float)sums[16 * (2 * th + tt) + 4 * gr + e]);
                }
#pragma unroll
                for (int i = 0; i < KH; ++i) {
                    const int j = KH * dh + i;
                    const v4f kv = widen(ak.column_of(ks, 2 * th + tt, j, tid));
                    const Frag<E> k0 = ak.cols_of(ks, 0, j, tid), k1 = ak.cols_of(ks, 1, j, tid);
                    v4f y = x2[tt][i], col = zero;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[e] *= -ga[e];
                        xdot[tt][e] += kv[e] * y[e];
                        y[e] *= be[e];
                    }
                    y = mma<E>(y, p0, k0);
                    if (th) y = mma<E>(y, p1, k1);
                    else col = mma<E>(col, p1, k0);
                    col = mma<E>(col, p3, k1);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dot[tt][e] += kv[e] * (y[e] - col[e]);
                    x2[tt][i] = y + col;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            leave_dots();
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (l == 4 * gr + e && mine < rows)
                    gbp[(int64_t)mine * a.Hv] =
                        (G)(mine < n ? whole_again((kScaled<E> ? rise * vd[e] : vd[e]) + dbs[mine] + (xdots[1][0][mine] + xdots[1][1][mine])) : 0.0f);
            __syncthreads();
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < KH; ++i) {
                    v4f y = x2[tt][i] + ex[((w * 2 + tt) * KH + i) * kWave + lane];
                    if constexpr (kScaled<E>)
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = whole_again(y[e]);
                    if constexpr (MANY) total[tt][i] += y;
                    else to_row(outk, tt, i, y);
                }
        }
    }
    if (MANY || n == 0) {
        __syncthreads();                              // (the last head's exchange has been read)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < KH; ++i) to_row(second ? outk : outq, tt, i, MANY ? total[MANY ? tt : 0][MANY ? i : 0] : zero);
    }
    __syncthreads();
    rows_out();
}

}  // namespace

hipError_t launch_delta_grad(int dtype, int gate_dtype, const void *q, const void *k, const void *v, const void *g, const void *beta, const void *go, void *gq,
                             void *gk, void *gv, void *gg, void *gbeta, const void *u, const void *r, const void *st, const void *ds,
                             const float *scales, int chunks, int cols, bool full, const DeltaArgs &a, const Steps (&gs)[3], hipStream_t s)
{
    dim3 grid;
    if (!spread(a.B * a.Hk * chunks, kThreads, grid)) return kNotTaken;
    const GradWs ws{u, r, st, ds, scales, chunks, cols};
    return by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        auto with = [&](auto *x) {
            using G = std::remove_pointer_t<decltype(x)>;
            auto go_ = [&](auto *kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, (const E *)q, (const E *)k, (const E *)v, (const G *)g, (const G *)beta,
                                   (const E *)go, (E *)gq, (E *)gk, (E *)gv, (G *)gg, (G *)gbeta, ws, a, gs[0], gs[1], gs[2]);
                return hipGetLastError();
            };
            auto shared = [&](auto many) {
                constexpr bool MANY = decltype(many)::value;
                if (a.Dk <= 64) return go_(full ? delta_grad_kernel<E, G, 64, MANY, true> : delta_grad_kernel<E, G, 64, MANY, false>);
                return go_(full ? delta_grad_kernel<E, G, 128, MANY, true> : delta_grad_kernel<E, G, 128, MANY, false>);
            };
            return a.Hv > a.Hk ? shared(std::true_type()) : shared(std::false_type());
        };
        return gate_dtype == dtype ? with((E *)nullptr) : with((float *)nullptr);
    });
}

}  // namespace sws

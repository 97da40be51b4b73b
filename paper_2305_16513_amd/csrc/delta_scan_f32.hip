// The passes of the gated delta rule that go from chunk to chunk, on fp32 storage: as delta_scan.hip has them, but with one wavefront per 16 columns
// of the state, which does everything; its operands are twice as wide, and two buffers of them would not fit LDS.
// A wavefront's products depend on each other, and the fp32 matrix instruction takes sixteen times the cycles of the 16-bit ones: bound by it.
// Five sequences of 777 tokens at most, six states each, Dk = 80, Dv = 72: forward 180 us, leaving states 100, backward 176.
#include "delta.h"

namespace sws {

namespace {

typedef float E;
constexpr int NW = 2;                                 // wavefronts, 16 columns each

template <int DK, int MODE, bool FULL>
__global__ __launch_bounds__(64 * NW) void delta_scan_kernel(const E *__restrict__ q, const E *__restrict__ k, const E *__restrict__ v,
                                                             E *__restrict__ o, float *__restrict__ state, ScanWs ws, DeltaArgs a)
{
    constexpr int NT = 64 * NW, W = 16 * NW, TRI = tri_bytes<E>();
    constexpr bool QUERIES = MODE != KEEP;
    constexpr int TRIS = MODE == KEEP ? 1 : 2, KINDS = MODE == FORWARD ? 2 : 3, FIRST = MODE == BACKWARD ? 1 : 0;   // loaded; there; the first that is loaded
    constexpr int TU = TRIS * TRI / 16, TN = (TU + NT - 1) / NT;
    typedef Tile<E, DK> Keys;
    typedef Tile<E, W> Values;
    __shared__ __align__(16) E ks[Keys::size(kChunk)], qs[QUERIES ? Keys::size(kChunk) : 8], vs[Values::size(kChunk)];
    const Keys at;
    const Values av;
    __shared__ __align__(16) v4u ts[TU];
    __shared__ __align__(16) float fs[3 * kChunk];
    const int w = threadIdx.x / kWave, lane = threadIdx.x % kWave, l = lane % 16, gr = lane / 16;
    const int64_t head = group_of(), b = group_of() / (unsigned)a.Hv;
    if (b >= a.B) return;
    const int h = (int)(head - b * a.Hv), hk = h / (a.Hv / a.Hk);
    const int col0 = blockIdx.y * W;                  // the workgroup's first column of the state
    int64_t len = tokens_of(a, b);
    const int64_t slot = a.slots ? a.slots[b] : b;
    if (state && a.slots && (slot < 0 || slot >= a.pool)) len = 0;
    float *const sp = state && (len > 0 || MODE == BACKWARD) ? state + (slot * a.Hv + h) * (int64_t)a.Dk * a.Dv : nullptr;
    const int my = col0 + 16 * w + l;                 // this lane's column
    const int chunks = chunks_of(len);

    v4f s[DK / 16];
#pragma unroll
    for (int i = 0; i < DK / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 16 * i + 4 * gr + e;
            s[i][e] = sp && r < a.Dk && my < a.Dv ? sp[(int64_t)r * a.Dv + my] : 0.0f;
        }

    const E *const kp = k + b * a.k.batch + hk * a.k.head, *const qp = q + b * a.q.batch + hk * a.q.head;
    const E *const vp = MODE == BACKWARD ? o + b * a.o.batch + h * a.o.head + col0 : v + b * a.v.batch + h * a.v.head + col0;
    const int64_t vstep = MODE == BACKWARD ? a.o.token : a.v.token;
    Rows<E, DK, NT, FULL> kr, qr;
    Rows<E, W, NT, FULL> vr;
    v4u tr[TN];
    float fr[3 * kChunk / NT + 1];
    auto fetch = [&](int c) {
        const int64_t t0 = (int64_t)c * kChunk;
        const int n = len - t0 < kChunk ? (int)(len - t0) : kChunk;
        kr.load(kp + t0 * a.k.token, a.k.token, n, a.Dk, threadIdx.x);
        if (QUERIES) qr.load(qp + t0 * a.q.token, a.q.token, n, a.Dk, threadIdx.x);
        vr.load(vp + t0 * vstep, vstep, n, a.Dv - col0, threadIdx.x);
        const v4u *tp = (const v4u *)(ws.tri + (head * ws.chunks + c) * (int64_t)(KINDS * TRI) + FIRST * TRI);
#pragma unroll
        for (int i = 0; i < TN; ++i)
            if (TU % NT == 0 || (int)threadIdx.x + i * NT < TU) tr[i] = tp[threadIdx.x + i * NT];
        const float *fp = ws.factors + (head * ws.chunks + c) * (int64_t)(3 * kChunk);
#pragma unroll
        for (int i = 0; i < 3 * kChunk / NT + 1; ++i)
            if ((int)threadIdx.x + i * NT < 3 * kChunk) fr[i] = fp[threadIdx.x + i * NT];
    };
    const E *const T = (const E *)ts, *const P = (const E *)ts + TRI / (int)sizeof(E);
    auto tri_frag = [&](const E *m, int at) { return get_pieces<E>(m, at); };

    // Of accumulators whose rows are tokens: the first row of the lane's column that is not finite, and rows from one on replaced
    auto first_of = [&](const v4f (&x)[4]) {
        int row = kChunk;
#pragma unroll
        for (int t = 3; t >= 0; --t)
#pragma unroll
            for (int e = 3; e >= 0; --e)
                if (!(__builtin_fabsf(x[t][e]) < __builtin_inff())) row = 16 * t + 4 * gr + e;
#pragma unroll
        for (int d = 16; d < kWave; d *= 2) {
            const int other = __shfl_xor(row, d);
            row = row < other ? row : other;
        }
        return row;
    };
    auto keep_before = [&](v4f (&x)[4], int row, float by) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * t + 4 * gr + e >= row) x[t][e] = by;
    };

    const int begin = MODE == BACKWARD ? chunks - 1 : 0, step = MODE == BACKWARD ? -1 : 1;
    if (chunks > 0) fetch(begin);
    for (int i = 0; i < chunks; ++i) {
        const int c = begin + i * step;
        const int64_t t0 = (int64_t)c * kChunk;
        __syncthreads();
        kr.store(ks, threadIdx.x);
        if (QUERIES) qr.store(qs, threadIdx.x);
        vr.store(vs, threadIdx.x);
#pragma unroll
        for (int j = 0; j < TN; ++j)
            if (TU % NT == 0 || (int)threadIdx.x + j * NT < TU) ts[threadIdx.x + j * NT] = tr[j];
#pragma unroll
        for (int j = 0; j < 3 * kChunk / NT + 1; ++j)
            if ((int)threadIdx.x + j * NT < 3 * kChunk) fs[threadIdx.x + j * NT] = fr[j];
        __syncthreads();
        if (i + 1 < chunks) fetch(c + step);

        const float all = fs[kChunk - 1];             // exp(G_63)
        const int64_t kept = (head * ws.chunks + c) * (ws.cols / 16) + (col0 / 16 + w);
        char *const up = MODE == FORWARD ? nullptr : (char *)ws.u + kept * Kept<E>::rows();
        Pieces<E> sx[DK / 32];
#pragma unroll
        for (int kb = 0; kb < DK / 32; ++kb) {
            sx[kb] = split<E>(s[2 * kb], s[2 * kb + 1]);
            if constexpr (MODE != FORWARD) Kept<E>::put((char *)ws.s + kept * Kept<E>::state(DK), kb, s[2 * kb], s[2 * kb + 1]);
        }

        auto factor = [&](int which, int t) { return *(const v4f *)(fs + which * kChunk + 16 * t + 4 * gr); };
        v4f x[4];                                     // K S: rows are tokens
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            x[t] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int kb = 0; kb < DK / 32; ++kb) x[t] = mma<E>(x[t], at.rows(ks, t, kb), sx[kb]);
        }
        if constexpr (MODE != BACKWARD) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {             // N
                const v4f vt = widen(av.column_of(vs, t, w)), gm = factor(0, t);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][e] = vt[e] - gm[e] * x[t][e];
            }
            auto solve = [&](const v4f (&n)[4]) {     // U
                const Pieces<E> n0 = split<E>(n[0], n[1]), n1 = split<E>(n[2], n[3]);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    x[t] = mma<E>(v4f{0, 0, 0, 0}, tri_frag(T, lower_at(t, 0)), n0);
                    if (t >= 2) x[t] = mma<E>(x[t], tri_frag(T, lower_at(t, 1)), n1);
                }
            };
            v4f n[4] = {x[0], x[1], x[2], x[3]};
            solve(n);
            int first = kChunk;                       // the first row of U that is not finite, of this lane's column
            if constexpr (MODE == FORWARD) {
                if (__any(!(__builtin_fabsf(x[3][0]) < __builtin_inff()))) {   // rows of N that are not finite have reached all of U's, times zeros of T: again without the first and those behind it
                    const int row = first_of(n);
                    keep_before(n, row, 0.0f);
                    solve(n);
                    keep_before(x, row, __builtin_nanf(""));
                }
                first = first_of(x);
            }
            if constexpr (MODE == KEEP) {
                Kept<E>::put(up, 0, x[0], x[1]);
                Kept<E>::put(up, 1, x[2], x[3]);
            } else {
                const bool some = __any(first < kChunk);
                v4f u[4] = {x[0], x[1], x[2], x[3]};
                if (some) keep_before(u, first, 0.0f);   // (as above, with the zeros of P)
                const Pieces<E> u0 = split<E>(u[0], u[1]), u1 = split<E>(u[2], u[3]);
                E *const op = o + b * a.o.batch + h * a.o.head + col0 + 16 * w + 4 * gr;
                const int there = a.Dv - (col0 + 16 * w + 4 * gr);
#pragma unroll
                for (int t = 0; t < 4; ++t) {         // O, rows are columns of the state
                    v4f y = {0, 0, 0, 0};
#pragma unroll
                    for (int kb = 0; kb < DK / 32; ++kb) y = mma<E>(y, sx[kb], at.rows(qs, t, kb));
                    const float gm = fs[16 * t + l];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] *= gm;
                    y = mma<E>(y, u0, tri_frag(P, lower_at(t, 0)));
                    if (t >= 2) y = mma<E>(y, u1, tri_frag(P, lower_at(t, 1)));
                    if (some)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (16 * t + l >= __shfl(first, 4 * gr + e)) y[e] = __builtin_nanf("");
                    const int64_t token = t0 + 16 * t + l;
                    if (token < a.T && there > 0) {
                        E *p = op + token * a.o.token;
                        typename Vec<E>::v4 out;
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[e] = token < len ? (E)(a.scale * y[e]) : (E)0.0f;   // (a row of zeros times a state that is not finite is not zero)
                        if constexpr (FULL) *(typename Vec<E>::v4 *)p = out;
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (e < there) p[e] = out[e];
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const v4f dl = factor(1, t);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][e] *= dl[e];
            }
            const Pieces<E> d0 = split<E>(x[0], x[1]), d1 = split<E>(x[2], x[3]);
#pragma unroll
            for (int j = 0; j < DK / 16; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[j][e] *= all;
                s[j] = mma<E>(s[j], at.cols(ks, 0, j), d0);
                s[j] = mma<E>(s[j], at.cols(ks, 1, j), d1);
            }
        } else {
            v4f y[4];                                 // exp(G) dO
            const Frag<E> o0 = av.cols_of(vs, 0, w), o1 = av.cols_of(vs, 1, w);
#pragma unroll
            for (int t = 0; t < 4; ++t) {             // dU
                v4f z = {0, 0, 0, 0};
                if (t < 2) z = mma<E>(z, tri_frag(P, upper_at(t, 0)), o0);
                z = mma<E>(z, tri_frag(P, upper_at(t, 1)), o1);
                const v4f dl = factor(1, t), gm = factor(0, t), vt = widen(av.column_of(vs, t, w));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[t][e] = dl[e] * x[t][e] + a.scale * z[e];
                    y[t][e] = a.scale * gm[e] * vt[e];
                }
            }
            const Pieces<E> u0 = split<E>(x[0], x[1]), u1 = split<E>(x[2], x[3]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {             // dR
                x[t] = v4f{0, 0, 0, 0};
                if (t < 2) x[t] = mma<E>(x[t], tri_frag(T, upper_at(t, 0)), u0);
                x[t] = mma<E>(x[t], tri_frag(T, upper_at(t, 1)), u1);
            }
            Kept<E>::put(up, 0, x[0], x[1]);
            Kept<E>::put(up, 1, x[2], x[3]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const v4f gm = factor(0, t), bt = factor(2, t);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[t][e] *= -gm[e] * bt[e];
            }
            const Pieces<E> r0 = split<E>(x[0], x[1]), r1 = split<E>(x[2], x[3]), y0 = split<E>(y[0], y[1]), y1 = split<E>(y[2], y[3]);
#pragma unroll
            for (int j = 0; j < DK / 16; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[j][e] *= all;
                s[j] = mma<E>(s[j], at.cols(ks, 0, j), r0);
                s[j] = mma<E>(s[j], at.cols(ks, 1, j), r1);
                s[j] = mma<E>(s[j], at.cols(qs, 0, j), y0);
                s[j] = mma<E>(s[j], at.cols(qs, 1, j), y1);
            }
        }
    }
    if (MODE != KEEP && sp && my < a.Dv)
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 16 * i + 4 * gr + e;
                if (r < a.Dk) sp[(int64_t)r * a.Dv + my] = s[i][e];
            }
    if constexpr (MODE == FORWARD) {                  // whole chunks of tokens that are not there
        const int width = a.Dv - col0 < W ? a.Dv - col0 : W;
        E *const op = o + b * a.o.batch + h * a.o.head + col0;
        for (int64_t t = (int64_t)chunks * kChunk + threadIdx.x / W; t < a.T; t += NT / W)
            if ((int)threadIdx.x % W < width) op[t * a.o.token + threadIdx.x % W] = (E)0.0f;
    }
}

template <int MODE>
hipError_t launch(const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws, const DeltaArgs &a, hipStream_t s)
{
    const int64_t heads = a.B * a.Hv;
    auto go = [&](auto dk) {
        constexpr int DK = decltype(dk)::value;
        // the gradients read whole blocks of 32 columns of what is kept
        const int cols = MODE == FORWARD ? a.Dv : ws.cols;
        const bool full = a.Dk == DK && a.Dv == cols && cols % (16 * NW) == 0 && full_rows<E>(a.q, DK, q) && full_rows<E>(a.k, DK, k) && full_rows<E>(a.v, 16 * NW, v) &&
                          full_rows<E>(a.o, 16 * NW, o);
        auto *kernel = full ? delta_scan_kernel<DK, MODE, true> : delta_scan_kernel<DK, MODE, false>;
        dim3 grid;
        if (!spread(heads, 64 * NW, grid, (unsigned)((cols + 16 * NW - 1) / (16 * NW)))) return kNotTaken;
        hipLaunchKernelGGL(kernel, grid, dim3(64 * NW), 0, s, (const E *)q, (const E *)k, (const E *)v, (E *)o, state, ws, a);
        return hipGetLastError();
    };
    using I64 = std::integral_constant<int, 64>;
    using I128 = std::integral_constant<int, 128>;
    return a.Dk <= 64 ? go(I64()) : go(I128());
}

}  // namespace

hipError_t launch_delta_scan_f32(int mode, const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws, const DeltaArgs &a,
                                 hipStream_t s)
{
    if (mode == FORWARD) return launch<FORWARD>(q, k, v, o, state, ws, a, s);
    if (mode == KEEP) return launch<KEEP>(q, k, v, o, state, ws, a, s);
    return launch<BACKWARD>(q, k, v, o, state, ws, a, s);
}

}  // namespace sws

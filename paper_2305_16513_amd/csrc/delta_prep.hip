// The first pass of the gated delta rule over chunks: what a chunk needs of its keys, queries and gates alone, for all chunks side by side.
//
//   T = (I + A)^-1,  A_ij = beta_i D_ij k_i.k_j (j < i),      P_ij = D_ij q_i.k_j (j <= i)
//
// T with its columns scaled by beta, and P (or, for the gradients, that, T^T and P^T) go to the workspace as operands in the order in which lanes take them, with the chunk's factors
// exp(G), exp(G_63 - G) and beta; in fp16 also the largest magnitudes of the chunk's values (and of their outputs' gradients), which the passes behind are scaled by.
//
// A workgroup takes one chunk of one value head.  Wavefront w multiplies tile row w of K K^T and Q K^T.  T in fp32: each
// wavefront inverts one 16 x 16 block of the diagonal, a lane a column, by substitution; blocks are then joined twice,
// X = -T_22 A_21 T_11, on the fp32 matrix instruction, first 16 and 16, then 32 and 32.  Sums of gates are taken in 64 bits: a
// decay is the exponential of the difference of two of them, which may be large beside it.
//
// Bound by its chain of small steps with barriers between them, so by how many chunks a CU holds: the matrices stand where K and Q were, 35 KB, and 16-bit types
// use 128 registers: four workgroups on a CU.  4096 chunks of bf16, Dk = 128: 75 us, for the gradients 84 (two workgroups took half as much again); what it reads and writes,
// 290 and 366 MB, takes 56 and 71 us.
#include "delta.h"

namespace sws {

namespace {

constexpr int kLd = 68;                               // floats of a row of the matrices: columns and rows of a tile on different banks

// A fp32 16 x 16 x 16 product of blocks in LDS (row r of x at x + r * kLd), and one whose right side is in accumulator layout
__device__ __forceinline__ v4f block_mul(v4f c, const float *x, const float *y)
{
    const int l = threadIdx.x % 16, g = threadIdx.x % kWave / 16;
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[l * kLd + 4 * g + e], y[(4 * g + e) * kLd + l], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ v4f block_mul(v4f c, const float *x, v4f y)
{
    const int l = threadIdx.x % 16, g = threadIdx.x % kWave / 16;
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[l * kLd + 4 * g + e], y[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ void block_put(float *to, v4f v, float sign)
{
    const int l = threadIdx.x % 16, g = threadIdx.x % kWave / 16;
#pragma unroll
    for (int e = 0; e < 4; ++e) to[(4 * g + e) * kLd + l] = sign * v[e];
}

template <class E, class G, int DK, bool FULL, bool GRAD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(E) == 4 ? 2 : 4))) void delta_prep_kernel(const E *__restrict__ q, const E *__restrict__ k, const G *__restrict__ g,
                                                         const G *__restrict__ beta, char *__restrict__ tri, float *__restrict__ factors, Magnitudes mg, int chunks,
                                                         DeltaArgs a)
{
    typedef Tile<E, DK> Keys;
    // K and Q, then in their place the two matrices
    constexpr int ROWS = Keys::size(kChunk), BYTES = 2 * (ROWS * (int)sizeof(E) > kChunk * kLd * 4 ? ROWS * (int)sizeof(E) : kChunk * kLd * 4);
    __shared__ __align__(16) char room[BYTES];
    E *const ks = (E *)room, *const qs = ks + ROWS;
    float *const A = (float *)room, *const P = A + kChunk * kLd;
    const Keys at;
    __shared__ double sums[kChunk];
    __shared__ float betas[kChunk];
    __shared__ unsigned tops[2][4];                   // of each wavefront
    __shared__ int broken;                            // A has numbers that are not finite
    const int w = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t head = group_of() / (unsigned)chunks, b = (unsigned)head / (unsigned)a.Hv;
    const int c = group_of() % (unsigned)chunks;
    if (b >= a.B) return;
    const int h = (int)(head - b * a.Hv), hk = h / (a.Hv / a.Hk);
    const int64_t t0 = (int64_t)c * kChunk, left = tokens_of(a, b) - t0;
    if (left <= 0) return;
    const int n = left < kChunk ? (int)left : kChunk;
    if constexpr (kScaled<E>) {                       // (the barriers in between are those of the matrices)
        unsigned top[2] = {0, 0};
        auto look = [&](const E *p, int64_t step, unsigned &to) {
            if (a.Dv % 8 == 0 && step % 8 == 0 && ((uintptr_t)p & 15) == 0) {      // eight elements a lane, whole rows a wavefront
                const int units = a.Dv / 8, many = kWave / units, r0 = lane / units, d = 8 * (lane % units);
                for (int r = w * many + r0; r < n && r0 < many; r += 4 * many) {
                    float f[8];
                    load8<true>(p + r * step + d, 8, f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const unsigned u = magnitude(f[e]);
                        to = to > u ? to : u;
                    }
                }
            } else
                for (int r = w; r < n; r += 4)
                    for (int d = lane; d < a.Dv; d += kWave) {
                        const unsigned u = magnitude((float)p[r * step + d]);
                        to = to > u ? to : u;
                    }
        };
        look((const E *)mg.v + b * a.v.batch + t0 * a.v.token + h * a.v.head, a.v.token, top[0]);
        if constexpr (GRAD) look((const E *)mg.go + b * a.o.batch + t0 * a.o.token + h * a.o.head, a.o.token, top[1]);
        if (c == 0) {
            auto look_at_state = [&](const float *s, int64_t place, unsigned &to) {
                const float *const p = s + (place * a.Hv + h) * (int64_t)a.Dk * a.Dv;
                for (int i = threadIdx.x; i < a.Dk * a.Dv; i += 256) {
                    const unsigned u = magnitude(p[i]);
                    to = to > u ? to : u;
                }
            };
            const int64_t place = a.slots ? a.slots[b] : b;
            if (mg.state && (!a.slots || (place >= 0 && place < a.pool))) look_at_state(mg.state, place, top[0]);
            if constexpr (GRAD)
                if (mg.gstate) look_at_state(mg.gstate, b, top[1]);
        }
#pragma unroll
        for (int i = 0; i < (GRAD ? 2 : 1); ++i) {
            top[i] = max_lanes(top[i]);
            if (lane == 0) tops[i][w] = top[i];
        }
    }
    {
        Rows<E, DK, 256, FULL> kr, qr;
        kr.load(k + b * a.k.batch + t0 * a.k.token + hk * a.k.head, a.k.token, n, a.Dk, threadIdx.x);
        qr.load(q + b * a.q.batch + t0 * a.q.token + hk * a.q.head, a.q.token, n, a.Dk, threadIdx.x);
        if (threadIdx.x == 0) broken = 0;
        if (w == 0) {
            const bool there = lane < n;
            const int64_t tk = t0 + lane;
            const float bt = there ? (float)beta[b * a.beta.batch + tk * a.beta.token + h * a.beta.head] : 0.0f;
            double s = there ? (double)gate((float)g[b * a.g.batch + tk * a.g.token + h * a.g.head]) : 0.0;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const double t = __shfl_up(s, d);
                if (lane >= d) s += t;
            }
            const double last = __shfl(s, kWave - 1);
            sums[lane] = s;
            betas[lane] = bt;
            float *f = factors + (head * chunks + c) * (3 * kChunk);
            f[lane] = decay<E>((float)s);
            f[kChunk + lane] = decay<E>((float)(last - s));
            f[2 * kChunk + lane] = bt;
        }
        kr.store(ks, threadIdx.x);
        qr.store(qs, threadIdx.x);
    }
    __syncthreads();
    if constexpr (kScaled<E>)
        if (threadIdx.x < (GRAD ? 2 : 1)) {
            const unsigned *t = tops[threadIdx.x], x = t[0] > t[1] ? t[0] : t[1], y = t[2] > t[3] ? t[2] : t[3];
            mg.tops[2 * (head * chunks + c) + threadIdx.x] = x > y ? x : y;
        }
    const int l = lane % 16, gr = lane / 16;
    v4f kk[4], qk[4];
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        kk[ct] = qk[ct] = v4f{0, 0, 0, 0};
        if (ct <= w) {
#pragma unroll
            for (int kb = 0; kb < DK / 32; ++kb) {
                const Frag<E> col = at.rows(ks, ct, kb);
                kk[ct] = Mx<E>::mma(kk[ct], at.rows(ks, w, kb), col);
                qk[ct] = Mx<E>::mma(qk[ct], at.rows(qs, w, kb), col);
            }
        }
    }
    double mine[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) mine[e] = sums[16 * w + 4 * gr + e];
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < 4; ++ct) {
        const int j = 16 * ct + l;
        const double theirs = sums[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * w + 4 * gr + e;
            const float d = i >= j ? decay<E>((float)(mine[e] - theirs)) : 0.0f;
            const float aij = i > j ? betas[i] * d * kk[ct][e] : 0.0f;
            A[i * kLd + j] = aij;
            P[i * kLd + j] = i >= j ? d * qk[ct][e] : 0.0f;
            if (!(__builtin_fabsf(aij) < INFINITY)) broken = 1;
        }
    }
    __syncthreads();
    if (broken) {                                     // (the same for all)
        // Row by row, a lane a column, over what is there alone: a row takes what is not finite from itself and rows before it.  (Products of whole blocks
        // would carry it, times zeros, to the others.)
        if (w == 0)
            for (int i = 0; i < kChunk; ++i) {
                float s = i == lane ? 1.0f : 0.0f;
                for (int m = 0; m < i; ++m) {
                    const float t = A[i * kLd + m] * A[m * kLd + lane];
                    if (m >= lane) s -= t;
                }
                __builtin_amdgcn_wave_barrier();      // (all lanes have read the row that they replace)
                A[i * kLd + lane] = s;
                __builtin_amdgcn_wave_barrier();
            }
        __syncthreads();
    } else {
    {                                                 // the diagonal's blocks
        float *blk = A + 16 * w * (kLd + 1), x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == l ? 1.0f : 0.0f;
#pragma unroll
            for (int m = 0; m < 16; ++m)
                if (m < i) s -= blk[i * kLd + m] * x[m];
            x[i] = s;
        }
        __syncthreads();
        if (gr == 0)
#pragma unroll
            for (int i = 0; i < 16; ++i) blk[i * kLd + l] = x[i];
    }
    __syncthreads();
    auto block = [&](int r, int s) { return A + 16 * r * kLd + 16 * s; };
    const v4f zero = {0, 0, 0, 0};
    {
        v4f y = zero;
        if (w < 2) y = block_mul(zero, block(2 * w + 1, 2 * w + 1), block_mul(zero, block(2 * w + 1, 2 * w), block(2 * w, 2 * w)));
        __syncthreads();
        if (w < 2) block_put(block(2 * w + 1, 2 * w), y, -1.0f);
    }
    __syncthreads();
    {
        const int bj = w & 1, xi = w >> 1;            // block (2 + xi, bj) is this wavefront's
        v4f x = zero;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            if (m > xi) continue;
            v4f y = zero;
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s >= bj) y = block_mul(y, block(2 + m, s), block(s, bj));
            x = block_mul(x, block(2 + xi, 2 + m), y);
        }
        __syncthreads();
        block_put(block(2 + xi, bj), x, -1.0f);
    }
    __syncthreads();
    }
    constexpr int TRI = tri_bytes<E>(), KINDS = GRAD ? 3 : 2;
    char *out = tri + (head * chunks + c) * (int64_t)(KINDS * TRI);
    for (int f = w; f < KINDS * kFrags; f += 4) {
        const int kind = f / kFrags, fa = f % kFrags;  // T beta, P;  T beta, T^T, P^T
        const float *M = kind == 0 || (GRAD && kind == 1) ? A : P;
        v4f lo, hi;
        if (!GRAD || kind == 0) {
            const int rt = fa < 2 ? fa : 2 + (fa - 2) / 2, kb = fa < 2 ? 0 : (fa - 2) & 1;
            const float *p = M + (16 * rt + l) * kLd + 32 * kb + 4 * gr;
            lo = *(const v4f *)p;
            hi = *(const v4f *)(p + 16);
            if (kind == 0) {
                const float *bt = betas + 32 * kb + 4 * gr;
#pragma unroll
                for (int e = 0; e < 4; ++e) {         // (zeros stay zeros whatever beta is)
                    const int below = 16 * rt + l - (32 * kb + 4 * gr + e);
                    lo[e] = below >= 0 ? lo[e] * bt[e] : 0.0f;
                    hi[e] = below >= 16 ? hi[e] * bt[16 + e] : 0.0f;
                }
            }
        } else {
            const int rt = fa < 4 ? fa / 2 : fa - 2, kb = fa < 4 ? fa & 1 : 1;
            const float *p = M + (32 * kb + 4 * gr) * kLd + 16 * rt + l;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = p[e * kLd];
                hi[e] = p[(16 + e) * kLd];
            }
        }
        put_pieces<E>((E *)(out + kind * TRI), fa, split<E>(lo, hi));
    }
}

}  // namespace

hipError_t launch_delta_prep(int dtype, int gate_dtype, const void *q, const void *k, const void *g, const void *beta, char *tri, float *factors,
                             const Magnitudes &mg, int chunks, bool full, bool grad, const DeltaArgs &a, hipStream_t s)
{
    dim3 grid;
    if (!spread(a.B * a.Hv * chunks, 256, grid)) return kNotTaken;
    return by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        auto with = [&](auto *u) {
            using G = std::remove_pointer_t<decltype(u)>;
            auto go = [&](auto *kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const E *)q, (const E *)k, (const G *)g, (const G *)beta, tri, factors, mg,
                                   chunks, a);
                return hipGetLastError();
            };
            if (a.Dk <= 64) {
                if (grad) return go(full ? delta_prep_kernel<E, G, 64, true, true> : delta_prep_kernel<E, G, 64, false, true>);
                return go(full ? delta_prep_kernel<E, G, 64, true, false> : delta_prep_kernel<E, G, 64, false, false>);
            }
            if (grad) return go(full ? delta_prep_kernel<E, G, 128, true, true> : delta_prep_kernel<E, G, 128, false, true>);
            return go(full ? delta_prep_kernel<E, G, 128, true, false> : delta_prep_kernel<E, G, 128, false, false>);
        };
        return gate_dtype == dtype ? with((E *)nullptr) : with((float *)nullptr);
    });
}

}  // namespace sws

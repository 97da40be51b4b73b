// The gated delta rule token by token: the form for decoding, where one token (or a few) of each sequence meets a state that lies in a pool.
//
// With w = S^T k and z = S^T q of the state before the token, everything follows from one pass over it:
//     u = beta (v - a w),   o = scale (a z + (q . k) u),   S <- a S + k u^T.
// Bound by HBM: the state is read and written once, in fp32, Dk Dv 8 bytes per value head, beside which the rest is nothing.  A workgroup
// holds Dk x W columns of one state in registers, W = 4 LANES: a lane four columns of every GROUPS-th row, so that LANES lanes
// read a row's W floats side by side.  w and z are summed within lanes, across the wavefront's rows and then through LDS.  128 columns
// where there are two workgroups of that for every CU; 32 where there are fewer, so that four times the workgroups share the latency of a read: one token, Dk =
// Dv = 128, 16 states 4.9 us against 7.3, 256 states 7.9 against 8.8, 512 states 12.9 against 11.5, 1024 states the same.
// The state stays in registers over all tokens of the call.  One token for 8192 such states, 1 GiB read and written: 216 us, 5.0 TB/s, what a copy reaches.
#include "delta.h"

namespace sws {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;                            // staged at a time

template <class E, class G, int DK, int LANES, bool FULL>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(const E *__restrict__ q, const E *__restrict__ k, const E *__restrict__ v,
                                                              const G *__restrict__ g, const G *__restrict__ beta, E *__restrict__ o,
                                                              float *__restrict__ pool, DeltaArgs a)
{
    constexpr int GROUPS = kThreads / LANES, ROWS = DK / GROUPS, W = 4 * LANES;
    static_assert(GROUPS * ROWS == DK && LANES <= 32, "");
    __shared__ float qs[kTokens][DK], ks[kTokens][DK], gs[kTokens], bs[kTokens], qk[kTokens];
    __shared__ v4f sums[2][2][4][LANES];              // in turn; w and z; of each wavefront
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, wave = threadIdx.x / kWave;
    const int64_t head = group_of(), b = group_of() / (unsigned)a.Hv;
    if (b >= a.B) return;
    const int h = (int)(head - b * a.Hv), hk = h / (a.Hv / a.Hk);
    const int c0 = blockIdx.y * W + 4 * lane, left = a.Dv - c0;       // columns of this lane
    int64_t len = tokens_of(a, b);
    const int64_t slot = a.slots ? a.slots[b] : b;
    if (pool && (slot < 0 || slot >= a.pool)) len = 0;                // a sequence without a place is left out
    float *sp = pool && len > 0 ? pool + (slot * a.Hv + h) * (int64_t)a.Dk * a.Dv : nullptr;
    v4f s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = group + GROUPS * i;
        s[i] = v4f{0, 0, 0, 0};
        if (sp && r < a.Dk && left > 0) {
            const float *p = sp + (int64_t)r * a.Dv + c0;
            if constexpr (FULL) s[i] = *(const v4f *)p;
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][e] = e < left ? p[e] : 0.0f;
        }
    }
    const E *qp = q + b * a.q.batch + hk * a.q.head, *kp = k + b * a.k.batch + hk * a.k.head, *vp = v + b * a.v.batch + h * a.v.head;
    const G *gp = g + b * a.g.batch + h * a.g.head, *bp = beta + b * a.beta.batch + h * a.beta.head;
    E *op = o + b * a.o.batch + h * a.o.head;
    int turn = 0;
    for (int64_t t0 = 0; t0 < len; t0 += kTokens) {
        const int n = len - t0 < kTokens ? (int)(len - t0) : kTokens;
        __syncthreads();
        for (int i = threadIdx.x; i < n * DK; i += kThreads) {
            const int t = i / DK, d = i % DK;
            const bool there = d < a.Dk;
            qs[t][d] = there ? (float)qp[(t0 + t) * a.q.token + d] : 0.0f;
            ks[t][d] = there ? (float)kp[(t0 + t) * a.k.token + d] : 0.0f;
        }
        if ((int)threadIdx.x < n) {
            gs[threadIdx.x] = expf((float)gp[(t0 + threadIdx.x) * a.g.token]);
            bs[threadIdx.x] = (float)bp[(t0 + threadIdx.x) * a.beta.token];
        }
        __syncthreads();
        for (int t = wave; t < n; t += 4) {
            float d = 0;
            for (int i = threadIdx.x % kWave; i < DK; i += kWave) d += qs[t][i] * ks[t][i];
            d = sum_lanes(d, kWave);
            if (threadIdx.x % kWave == 0) qk[t] = d;
        }
        for (int t = 0; t < n; ++t) {
            v4f vt = {0, 0, 0, 0};
            if (left > 0) {
                const E *p = vp + (t0 + t) * a.v.token + c0;
#pragma unroll
                for (int e = 0; e < 4; ++e) vt[e] = FULL || e < left ? (float)p[e] : 0.0f;
            }
            v4f w = {0, 0, 0, 0}, z = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const float kr = ks[t][group + GROUPS * i], qr = qs[t][group + GROUPS * i];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] += kr * s[i][e];
                    z[e] += qr * s[i][e];
                }
            }
#pragma unroll
            for (int d = LANES; d < kWave; d <<= 1)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] += __shfl_xor(w[e], d);
                    z[e] += __shfl_xor(z[e], d);
                }
            if (threadIdx.x % kWave < LANES) {
                sums[turn][0][wave][lane] = w;
                sums[turn][1][wave][lane] = z;
            }
            __syncthreads();
            const v4f *sw = &sums[turn][0][0][lane], *sz = &sums[turn][1][0][lane];
            w = (sw[0] + sw[LANES]) + (sw[2 * LANES] + sw[3 * LANES]);
            z = (sz[0] + sz[LANES]) + (sz[2 * LANES] + sz[3 * LANES]);
            turn ^= 1;
            const float at = gs[t], bt = bs[t], d = qk[t];
            v4f u;
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = bt * (vt[e] - at * w[e]);
            if (group == 0 && left > 0) {
                E *p = op + (t0 + t) * a.o.token + c0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (FULL || e < left) p[e] = (E)(a.scale * (at * z[e] + d * u[e]));
            }
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const float kr = ks[t][group + GROUPS * i];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][e] = at * s[i][e] + kr * u[e];
            }
        }
    }
    if (sp && left > 0)
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = group + GROUPS * i;
            if (r >= a.Dk) continue;
            float *p = sp + (int64_t)r * a.Dv + c0;
            if constexpr (FULL) *(v4f *)p = s[i];
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) p[e] = s[i][e];
        }
    if (left > 0 && group == 0)                       // tokens that are not there
        for (int64_t t = len; t < a.T; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (FULL || e < left) op[t * a.o.token + c0 + e] = (E)0.0f;
}

}  // namespace

hipError_t launch_delta_step(int dtype, int gate_dtype, const void *q, const void *k, const void *v, const void *g, const void *beta, void *o,
                             float *pool, const DeltaArgs &a, hipStream_t s)
{
    const int64_t heads = a.B * a.Hv;
    const bool wide = heads * ((a.Dv + 127) / 128) >= 2 * device_cus();
    dim3 grid;
    if (!spread(heads, kThreads, grid, (unsigned)((a.Dv + (wide ? 127 : 31)) / (wide ? 128 : 32)))) return kNotTaken;
    const bool full = a.Dv % 4 == 0 && ((uintptr_t)pool & 15) == 0;
    return by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        auto with = [&](auto *u) {
            using G = std::remove_pointer_t<decltype(u)>;
            auto go = [&](auto *kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, (const E *)q, (const E *)k, (const E *)v, (const G *)g, (const G *)beta, (E *)o,
                                   pool, a);
                return hipGetLastError();
            };
            if (a.Dk <= 64) {
                if (wide) return go(full ? delta_step_kernel<E, G, 64, 32, true> : delta_step_kernel<E, G, 64, 32, false>);
                return go(full ? delta_step_kernel<E, G, 64, 8, true> : delta_step_kernel<E, G, 64, 8, false>);
            }
            if (wide) return go(full ? delta_step_kernel<E, G, 128, 32, true> : delta_step_kernel<E, G, 128, 32, false>);
            return go(full ? delta_step_kernel<E, G, 128, 8, true> : delta_step_kernel<E, G, 128, 8, false>);
        };
        return gate_dtype == dtype ? with((E *)nullptr) : with((float *)nullptr);
    });
}

}  // namespace sws

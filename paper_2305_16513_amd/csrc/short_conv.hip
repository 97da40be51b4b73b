// The short causal convolution of a language model's layer, on rows of tokens: per channel a sliding dot product over the k last
// tokens, then bias, activation and, for the first channels, a scaling of every head to length one:
//
//   p[b,t,c] = bias[c] + sum_j f[c,j] x[b, t-k+1+j, c],   a = p or p * sigmoid(p),   y = a * rsqrt(sum over the head of a^2 + eps) or a
//
// Tokens in front of the first are the sequence's context (k - 1 tokens in a pool, replaced by the last ones) or zeros.  Gradients, with
// i the head's factor:  ga = i (gy - y * sum of y gy),  gp = ga da/dp,  gx[t] = sum_j f[j] gp[t+k-1-j],  gf[j] = sum over t of gp[t] x[t-k+1+j],
// gbias = sum of gp.
//
// Forward bound by HBM, backward by its arithmetic.  A lane owns eight channels (16 bytes of a 16-bit row) and a run of tokens, which slide through its registers with the
// taps, so that a token is read once per run; the k - 1 tokens that two runs share come from the caches.  A head's sum of squares goes across the
// lanes that hold it (a power of two of them, idle ones among them where a head has fewer groups of eight).  The backward pass computes p
// again instead of reading it.  Sums over tokens leave as one partial row per run and are added in a fixed order.
//
// [4, 4096, 6144] bf16, four taps, 4096 channels in heads of 128 to length one: forward 94 us for 403 MB (4.3 TB/s; a copy of 1 GiB: 5.1), vector units busy for 69 % of them;
// gradients 206 us for 604 MB, arithmetic more than memory: a head's two sums, eight sigmoids and their slopes per token keep the vector units busy for 68 % of the time, with 1.6
// wavefronts on a SIMD (214 registers, two workgroups on a CU).  64 sequences' single tokens: 7 us, the launch and latency.  Rows that are no multiple of eight channels, or not at
// multiples of 16 bytes, are taken element by element: 6143 channels, none normed, 241 and 324 us (6144: 92 and 149).
#include "seq.h"

namespace sws {

namespace {

constexpr int kThreads = 256;
constexpr int kPlaces = 4, kGradPlaces = 2;           // workgroups that a CU's registers hold (116 and 214 of a thread's, four taps)

struct ShortConvArgs {
    int64_t B, T;
    int64_t xb, xt, yb, yt, gxb, gxt;                 // elements from one sequence to the next, from one token to the next
    int C, unit, heads, normed;                       // channels; channels of a head, heads, how many of them are normed
    int lanes;                                        // per head: a power of two
    int silu, run, runs;                              // tokens of a run, runs of a sequence
    int64_t pool;                                     // places of the pool
    float eps;
};

// Where this thread works: its channels, its run, and how much of a head it holds.
struct Place {
    int64_t b;
    int c0, left, head, run;
    bool live;
};

__device__ __forceinline__ Place place_of(const ShortConvArgs &a)
{
    Place p;
    const int per = kThreads / a.lanes, group = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes;
    p.head = blockIdx.x * per + group;
    const unsigned at = blockIdx.z * gridDim.y + blockIdx.y;      // (the last of z may reach beyond the last sequence)
    p.run = at % a.runs;
    p.b = at / a.runs;
    p.live = p.head < a.heads;
    p.c0 = p.head * a.unit + 8 * lane;
    const int in_head = a.unit - 8 * lane, in_row = a.C - p.c0;
    p.left = p.live ? (in_head < in_row ? in_head : in_row) : 0;
    if (p.left < 0) p.left = 0;
    if (p.left == 0) p.c0 = 0;
    return p;
}

// f[j][e], bias[e] of the thread's channels; zeros beyond them.  (The eight channels' taps lie side by side.)
template <int K, bool FULL>
__device__ __forceinline__ void load_taps(const float *__restrict__ w, const float *__restrict__ bias, const Place &p, float (&f)[K][8], float (&b)[8])
{
    if constexpr (FULL) {
        if (p.left <= 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int j = 0; j < K; ++j) f[j][e] = 0;
                b[e] = 0;
            }
            return;
        }
        v4f t[2 * K];
#pragma unroll
        for (int i = 0; i < 2 * K; ++i) t[i] = *(const v4f *)(w + (int64_t)p.c0 * K + 4 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int j = 0; j < K; ++j) f[j][e] = t[(e * K + j) / 4][(e * K + j) % 4];
        if (bias) load8<true>(bias + p.c0, 8, b);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = 0;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int j = 0; j < K; ++j) f[j][e] = e < p.left ? w[(int64_t)(p.c0 + e) * K + j] : 0.0f;
        b[e] = bias && e < p.left ? bias[p.c0 + e] : 0.0f;
    }
}

template <bool FULL, class E>
__device__ __forceinline__ void load_token(const E *base, int64_t t, int64_t stride, const Place &p, bool there, float (&v)[8])
{
    if (there && p.left > 0) load8<FULL>(base + t * stride + p.c0, p.left, v);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0;
}

template <bool FULL, class E>
__device__ __forceinline__ typename Vec<E>::v8 fetch_token(const E *base, int64_t t, int64_t stride, const Place &p, bool there)
{
    if (there && p.left > 0) return fetch8<FULL>(base + t * stride + p.c0, p.left);
    return typename Vec<E>::v8{};
}

template <class E, int K, bool FULL>
__global__ __launch_bounds__(kThreads) void short_conv_kernel(const E *__restrict__ x, const float *__restrict__ w, const float *__restrict__ bias,
                                                              E *state, const int *__restrict__ slots, const int *__restrict__ lengths,
                                                              E *__restrict__ y, ShortConvArgs a)
{
    constexpr int H = K - 1;
    const Place p = place_of(a);
    if (p.b >= a.B) return;
    int64_t len = lengths ? lengths[p.b] : a.T;
    len = len < 0 ? 0 : len < a.T ? len : a.T;
    int64_t slot = slots ? slots[p.b] : p.b;
    const bool known = !state || (slot >= 0 && slot < a.pool);   // a sequence without a place is left out
    if (!known) len = 0;
    const int64_t t0 = (int64_t)p.run * a.run, t1 = t0 + a.run < a.T ? t0 + a.run : a.T;
    float f[K][8], bs[8];
    load_taps<K, FULL>(w, bias, p, f, bs);
    const E *xp = x + p.b * a.xb;
    E *yp = y + p.b * a.yb + p.c0;
    E *sp = state && known ? state + slot * H * a.C : nullptr;
    float win[K][8];                                  // win[j]: token t - K + 1 + j
#pragma unroll
    for (int j = 0; j < H; ++j) {
        const int64_t t = t0 - H + j;
        if (t < 0) load_token<FULL>(sp, t + H, a.C, p, sp != nullptr, win[j]);
        else load_token<FULL>(xp, t, a.xt, p, t < len, win[j]);
    }
    if (sp && p.run == 0 && p.left > 0) {             // the context's place gets the last K - 1 of its tokens and the sequence's
        float last[H > 0 ? H : 1][8];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            const int64_t t = len - H + j;
            load_token<FULL>(t < 0 ? (const E *)sp : xp, t < 0 ? t + H : t, t < 0 ? (int64_t)a.C : a.xt, p, true, last[j]);
        }
#pragma unroll
        for (int j = 0; j < H; ++j) store8<FULL>(sp + (int64_t)j * a.C + p.c0, p.left, last[j]);
    }
    const bool normed = p.head < a.normed;
    typename Vec<E>::v8 next[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = fetch_token<FULL>(xp, t0 + i, a.xt, p, t0 + i < t1 && t0 + i < len);
    for (int64_t t = t0; t < t1; t += 4) {
        typename Vec<E>::v8 in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            in[i] = next[i];
            next[i] = fetch_token<FULL>(xp, t + 4 + i, a.xt, p, t + 4 + i < t1 && t + 4 + i < len);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float o[8], sum = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                win[H][e] = (float)in[i][e];
                o[e] = bs[e];
#pragma unroll
                for (int j = 0; j < K; ++j) o[e] += f[j][e] * win[j][e];
                if (a.silu) o[e] *= sigmoid<E>(o[e]);
                sum += e < p.left ? o[e] * o[e] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < H; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) win[j][e] = win[j + 1][e];
            if (a.normed) {
                sum = sum_lanes(sum, a.lanes);
                const float inv = normed ? 1.0f / sqrtf(sum + a.eps) : 1.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] *= inv;
            }
            if (t + i < t1 && p.left > 0) {
                if (t + i >= len)
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = 0;
                store8<FULL>(yp + (t + i) * a.yt, p.left, o);
            }
        }
    }
}

template <class E, int K, bool FULL>
__global__ __launch_bounds__(kThreads) void short_conv_grad_kernel(const E *__restrict__ x, const float *__restrict__ w, const float *__restrict__ bias,
                                                                   const int *__restrict__ lengths, const E *__restrict__ gy, E *__restrict__ gx,
                                                                   float *__restrict__ part, ShortConvArgs a)
{
    constexpr int H = K - 1;
    const Place p = place_of(a);
    if (p.b >= a.B) return;
    int64_t len = lengths ? lengths[p.b] : a.T;
    len = len < 0 ? 0 : len < a.T ? len : a.T;
    const int64_t t0 = (int64_t)p.run * a.run, t1 = t0 + a.run < a.T ? t0 + a.run : a.T;
    float f[K][8], bs[8], gf[K][8] = {}, gb[8] = {};
    load_taps<K, FULL>(w, bias, p, f, bs);
    const E *xp = x + p.b * a.xb, *gp0 = gy + p.b * a.yb;
    E *gxp = gx + p.b * a.gxb + p.c0;
    float win[K][8], gp[K][8];                        // tokens t - K + 1 ..., gradients of p at the same ones
#pragma unroll
    for (int j = 0; j < H; ++j) {
        load_token<FULL>(xp, t0 - H + j, a.xt, p, t0 - H + j >= 0 && t0 - H + j < len, win[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) gp[j][e] = 0;
    }
    const bool normed = p.head < a.normed;
    // token t's gradient of p, then gx of token t - K + 1, whose last tap it was: K - 1 tokens of the next run too
    typename Vec<E>::v8 nx[2], ng[2];
    auto fetch = [&](int64_t t, int i) {
        const bool there = t < t1 + H && t < len;
        nx[i] = fetch_token<FULL>(xp, t, a.xt, p, there);
        ng[i] = fetch_token<FULL>(gp0, t, a.yt, p, there);
    };
    fetch(t0, 0);
    fetch(t0 + 1, 1);
    for (int64_t t = t0; t < t1 + H; t += 2) {
        typename Vec<E>::v8 in[2], gin[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            in[i] = nx[i];
            gin[i] = ng[i];
            fetch(t + 2 + i, i);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float act[8], sl[8], gi[8], ss = 0, dot = 0;         // activation, its slope
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                win[H][e] = (float)in[i][e];
                gi[e] = (float)gin[i][e];
                float o = bs[e];
#pragma unroll
                for (int j = 0; j < K; ++j) o += f[j][e] * win[j][e];
                const float s = a.silu ? sigmoid<E>(o) : 1.0f;
                act[e] = o * s;
                sl[e] = a.silu ? s + act[e] * (1.0f - s) : 1.0f;
                ss += e < p.left ? act[e] * act[e] : 0.0f;
                dot += act[e] * gi[e];
            }
            if (a.normed) {
                ss = sum_lanes(ss, a.lanes);
                dot = sum_lanes(dot, a.lanes);
                if (normed) {
                    const float inv = 1.0f / sqrtf(ss + a.eps), d = dot * inv * inv;
#pragma unroll
                    for (int e = 0; e < 8; ++e) gi[e] = inv * (gi[e] - act[e] * d);
                }
            }
            const bool real = t + i < len && t + i < t1 + H;
#pragma unroll
            for (int e = 0; e < 8; ++e) gp[H][e] = real ? gi[e] * sl[e] : 0.0f;
            if (real && t + i < t1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    gb[e] += gp[H][e];
#pragma unroll
                    for (int j = 0; j < K; ++j) gf[j][e] += gp[H][e] * win[j][e];
                }
            }
            const int64_t out = t + i - H;            // gp[j] is token out + j's
            if (out >= t0 && out < t1 && p.left > 0) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = 0;
#pragma unroll
                    for (int j = 0; j < K; ++j) o[e] += f[H - j][e] * gp[j][e];
                    if (out >= len) o[e] = 0;
                }
                store8<FULL>(gxp + out * a.gxt, p.left, o);
            }
#pragma unroll
            for (int j = 0; j < H; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    win[j][e] = win[j + 1][e];
                    gp[j][e] = gp[j + 1][e];
                }
        }
    }
    float *out = part + (p.b * a.runs + p.run) * (int64_t)a.C * (K + 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e >= p.left) continue;
#pragma unroll
        for (int j = 0; j < K; ++j) out[(int64_t)(p.c0 + e) * K + j] = gf[j][e];
        out[(int64_t)a.C * K + p.c0 + e] = gb[e];
    }
}

template <class F>
hipError_t by_taps(int k, F &&f)
{
    switch (k) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    case 4: return f(std::integral_constant<int, 4>());
    case 5: return f(std::integral_constant<int, 5>());
    case 6: return f(std::integral_constant<int, 6>());
    case 7: return f(std::integral_constant<int, 7>());
    case 8: return f(std::integral_constant<int, 8>());
    }
    return kNotTaken;
}

// Heads of `unit` channels (0: none are normed, and channels lie side by side: 512 of them are then a wavefront's) and runs of tokens, of which `slots`
// workgroups a CU are at work at once: a run costs its tokens and some eight more (those that it shares with its neighbours, the taps, what a workgroup takes to start),
// and a last round of few workgroups as much as a full one ([4, 4096, 6144], gradients: 768 workgroups of 64 tokens, two rounds on 512 places, 198 us; 492 of 100 tokens, one
// round, 189 us; shortest runs of both).
// No run is shorter than 8 unless it is the only one: the context, which the first run replaces, is then no other run's to read (k <= 8).
void plan(ShortConvArgs &a, int unit, int unit_channels, int slots)
{
    a.unit = unit_channels ? unit : 512;
    a.heads = (a.C + a.unit - 1) / a.unit;
    a.normed = unit_channels / a.unit;
    a.lanes = 1;
    while (a.lanes * 8 < a.unit) a.lanes *= 2;
    const int per = kThreads / a.lanes;
    const int64_t across = (a.heads + per - 1) / per * a.B, places = (int64_t)slots * device_cus();
    int64_t best = 0;
    a.run = 8;
    for (int run = 8; run <= 128; run += 4) {
        const int64_t cost = (across * ((a.T + run - 1) / run) + places - 1) / places * (run + 8);
        if (!best || cost < best) best = cost, a.run = run;
    }
    if (a.run > a.T) a.run = (int)a.T;
    a.runs = (int)((a.T + a.run - 1) / a.run);
}

// Runs of all sequences in y and z, at most 65535 in each
bool grid_of(const ShortConvArgs &a, dim3 &grid)
{
    const int per = kThreads / a.lanes;
    const int64_t gx = (a.heads + per - 1) / per, n = a.B * a.runs;
    if (n > 0x7fffffff) return false;
    const int64_t gz = (n + 65534) / 65535, gy = (n + gz - 1) / gz;
    grid = dim3((unsigned)gx, (unsigned)gy, (unsigned)gz);
    return true;
}

}  // namespace

int64_t short_conv_grad_bytes(int64_t B, int64_t T, int C, int k, int unit, int unit_channels)
{
    ShortConvArgs a{};
    a.B = B, a.T = T, a.C = C;
    plan(a, unit, unit_channels, kGradPlaces);
    return 4 * B * a.runs * C * (k + 1);
}

hipError_t launch_short_conv(int dtype, const void *x, const float *w, const float *bias, void *state, const int *slots, const int *lengths, void *y,
                             int64_t B, int64_t T, int C, int k, int64_t xb, int64_t xt, int64_t yb, int64_t yt, int64_t pool, int act, int unit,
                             int unit_channels, float eps, hipStream_t s)
{
    ShortConvArgs a{};
    a.B = B, a.T = T, a.C = C, a.xb = xb, a.xt = xt, a.yb = yb, a.yt = yt, a.silu = act == SWS_ACT_SILU, a.pool = pool, a.eps = eps;
    plan(a, unit, unit_channels, kPlaces);
    dim3 grid;
    if (!grid_of(a, grid)) return kNotTaken;
    const bool full = C % 8 == 0 && a.unit % 8 == 0 && xb % 8 == 0 && xt % 8 == 0 && yb % 8 == 0 && yt % 8 == 0 && sixteen({x, state, y, w, bias});
    return by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        return by_taps(k, [&](auto taps) {
            constexpr int K = decltype(taps)::value;
            auto *kernel = full ? short_conv_kernel<E, K, true> : short_conv_kernel<E, K, false>;
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, (const E *)x, w, bias, (E *)state, slots, lengths, (E *)y, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_short_conv_grad(int dtype, const void *x, const float *w, const float *bias, const int *lengths, const void *gy, void *gx, float *gw,
                                  float *gbias, int64_t B, int64_t T, int C, int k, int64_t xb, int64_t xt, int64_t gyb, int64_t gyt, int64_t gxb,
                                  int64_t gxt, int act, int unit, int unit_channels, float eps, Workspace ws, hipStream_t s)
{
    ShortConvArgs a{};
    a.B = B, a.T = T, a.C = C, a.xb = xb, a.xt = xt, a.yb = gyb, a.yt = gyt, a.gxb = gxb, a.gxt = gxt, a.silu = act == SWS_ACT_SILU, a.eps = eps;
    const bool none = B == 0 || T == 0;               // the sums are zero then
    dim3 grid;
    if (!none) {
        plan(a, unit, unit_channels, kGradPlaces);
        if (!grid_of(a, grid)) return kNotTaken;
    }
    const bool full = C % 8 == 0 && a.unit % 8 == 0 && xb % 8 == 0 && xt % 8 == 0 && gyb % 8 == 0 && gyt % 8 == 0 && gxb % 8 == 0 && gxt % 8 == 0 &&
                      sixteen({x, gy, gx, w, bias});
    float *part = (float *)ws.p;
    hipError_t e = none ? hipSuccess : by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        return by_taps(k, [&](auto taps) {
            constexpr int K = decltype(taps)::value;
            auto *kernel = full ? short_conv_grad_kernel<E, K, true> : short_conv_grad_kernel<E, K, false>;
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, (const E *)x, w, bias, lengths, (const E *)gy, (E *)gx, part, a);
            return hipGetLastError();
        });
    });
    const int parts = none ? 0 : (int)(B * a.runs);
    const int64_t stride = (int64_t)C * (k + 1);
    if (e == hipSuccess) e = launch_column_sums(part, gw, gbias, (int64_t)C * k, parts, stride, gbias ? stride : (int64_t)C * k, s);
    return e;
}

}  // namespace sws

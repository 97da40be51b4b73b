// The norms of a block of a language model, forward and gradients, on fp32, bf16 and fp16 storage with fp32 arithmetic:
//
//   before it   h = r + gain * x (gain per column, absent: 1; x absent: h = r),   n = h * i * w,   i = 1 / sqrt(mean(h^2) + eps)
//   behind it   y = x * i * w * z * sigmoid(z),   per head of D columns
//
// Gradients, with hn = h * i:   gh' = gh + i * (gn w - hn * mean(gn w hn)),   gr = gh',   gx = gain gh',   gw = sum over rows of gn hn,
// ggain = sum over rows of gh' x.  h is computed again from r and x, so that nothing is rounded on the way.
//
// Bound by HBM: one read of every input, one write of every output.  A row is held in registers by NT lanes (8 elements at a time, NV
// times), between its sum and its outputs; heads of up to 256 columns take 8 - 32 lanes, so that a wavefront holds several, rows of more than
// 2048 columns the whole workgroup.  Column sums stay in registers over all rows of a workgroup, leave as one partial row of it and are
// added by column_sums_kernel in a fixed order.
//
// [16384, 4096] bf16, x and gain there: forward 101 us for 537 MB, gradients 191 us for 805 MB (4.2 TB/s; a copy of 1 GiB: 5.1); [16384, 16 heads of 128]
// bf16: 39 us for 201 MB, gradients 65 us for 336 MB.  Eight rows of 1800: 6 us, the launch and a read's latency.  Rows that are no multiple of eight columns, or not at multiples of 16
// bytes, are taken element by element: [16384, 4095] 461 and 805 us, [16384, 16 heads of 127] 134 and 257 us.
#include "seq.h"

namespace sws {

namespace {

constexpr int kThreads = 256;

// The sum of v over the NT threads of a row.  NT = 256: all threads of the workgroup arrive here.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float *lds, int &turn)
{
    constexpr int n = NT < kWave ? NT : kWave;
    v = sum_lanes(v, n);
    if constexpr (NT > kWave) {
        float *at = lds + 4 * turn;                   // two places in turn: a thread may still read the last sum
        turn ^= 1;
        if (threadIdx.x % kWave == 0) at[threadIdx.x / kWave] = v;
        __syncthreads();
        v = (at[0] + at[1]) + (at[2] + at[3]);
    }
    return v;
}

// Column sums of a workgroup's row groups (kThreads / NT of them) to one partial row: `s` of every thread, by way of LDS.
template <int NT, int NV>
__device__ __forceinline__ void leave_sums(const float (&s)[NV][8], float *__restrict__ out, int width, float *lds)
{
    constexpr int GROUPS = kThreads / NT;
    const int lane = threadIdx.x % NT;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = (i * NT + lane) * 8;
        if constexpr (GROUPS == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c0 + e < width) out[c0 + e] = s[i][e];
        } else {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[e * kThreads + threadIdx.x] = s[i][e];
            __syncthreads();
            for (int q = threadIdx.x; q < NT * 8; q += kThreads) {
                const int e = q & 7, l = q >> 3, c = (i * NT + l) * 8 + e;
                if (c >= width) continue;
                float t = lds[e * kThreads + l];
                for (int g = 1; g < GROUPS; ++g) t += lds[e * kThreads + g * NT + l];
                out[c] = t;
            }
        }
    }
}

struct NormArgs {
    int64_t rows;
    int width;
    float eps, inv_width;
};

template <class E, int NT, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void norm_add_kernel(const E *__restrict__ r, const E *__restrict__ x, const float *__restrict__ gain,
                                                            const float *__restrict__ w, E *__restrict__ h, E *__restrict__ n, NormArgs a)
{
    __shared__ float lds[8];
    int turn = 0;
    const int lane = threadIdx.x % NT;
    const int64_t row = (int64_t)group_of() * (kThreads / NT) + threadIdx.x / NT;
    const bool live = row < a.rows;                   // (no return: shuffles and barriers are everybody's)
    const int64_t base = live ? row * a.width : 0;
    float v[NV][8], sum = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
        if (FULL && left <= 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0;
            continue;
        }
        load8<FULL>(r + base + c0, left, v[i]);
        if (x) {
            float t[8], g[8];
            load8<FULL>(x + base + c0, left, t);
            if (gain) load8<FULL>(gain + c0, left, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = gain ? v[i][e] + g[e] * t[e] : v[i][e] + t[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[i][e] * v[i][e];
    }
    const float inv = 1.0f / sqrtf(row_sum<NT>(sum, lds, turn) * a.inv_width + a.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
        if (left <= 0) continue;
        float t[8];
        load8<FULL>(w + c0, left, t);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= v[i][e] * inv;
        if (h) store8<FULL>(h + base + c0, left, v[i]);
        store8<FULL>(n + base + c0, left, t);
    }
}

template <class E, int NT, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void norm_add_grad_kernel(const E *__restrict__ r, const E *__restrict__ x, const float *__restrict__ gain,
                                                                 const float *__restrict__ w, const E *__restrict__ gn, const E *__restrict__ gh,
                                                                 E *__restrict__ gr, E *__restrict__ gx, float *__restrict__ part, NormArgs a)
{
    __shared__ float lds[NT == kThreads ? 8 : 8 * kThreads];
    int turn = 0;
    constexpr int GROUPS = kThreads / NT;
    const int lane = threadIdx.x % NT;
    float sw[NV][8] = {}, sg[NV][8] = {};
    // the next row of this workgroup is in flight during this one
    typename Vec<E>::v8 nr[NV], nx[NV], nd[NV], ng[NV];
    auto fetch = [&](int64_t row) {
        const bool live = row < a.rows;
        const int64_t base = live ? row * a.width : 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
            nr[i] = nx[i] = nd[i] = ng[i] = typename Vec<E>::v8{};
            if (left <= 0) continue;
            nr[i] = fetch8<FULL>(r + base + c0, left);
            nd[i] = fetch8<FULL>(gn + base + c0, left);
            if (x) nx[i] = fetch8<FULL>(x + base + c0, left);
            if (gh) ng[i] = fetch8<FULL>(gh + base + c0, left);
        }
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    fetch((int64_t)blockIdx.x * GROUPS + threadIdx.x / NT);
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < a.rows; first += step) {
        const int64_t row = first + threadIdx.x / NT;
        const bool live = row < a.rows;
        const int64_t base = live ? row * a.width : 0;
        float v[NV][8], xs[NV][8], d[NV][8], sum = 0, dot = 0;
        typename Vec<E>::v8 h8[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = (float)nr[i][e], xs[i][e] = (float)nx[i][e], d[i][e] = (float)nd[i][e];
            h8[i] = ng[i];
            if (left <= 0) continue;                  // (zeros)
            if (x) {
                float g[8];
                if (gain) load8<FULL>(gain + c0, left, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = gain ? v[i][e] + g[e] * xs[i][e] : v[i][e] + xs[i][e];
            }
            float t[8];
            load8<FULL>(w + c0, left, t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum += v[i][e] * v[i][e];
                dot += d[i][e] * t[e] * v[i][e];
            }
        }
        fetch(row + step);
        // both sums in one go: of the squares, and of gn w h, which is the one with hn divided by i
        float inv, mean;
        if constexpr (NT > kWave) {
            sum = row_sum<kWave>(sum, lds, turn);
            dot = row_sum<kWave>(dot, lds, turn);
            // two places in turn; a wavefront's two sums side by side
            __shared__ float both[2][8];
            float *at = both[turn];
            turn ^= 1;
            if (threadIdx.x % kWave == 0) {
                at[threadIdx.x / kWave] = sum;
                at[4 + threadIdx.x / kWave] = dot;
            }
            __syncthreads();
            sum = (at[0] + at[1]) + (at[2] + at[3]);
            dot = (at[4] + at[5]) + (at[6] + at[7]);
        } else {
            sum = row_sum<NT>(sum, lds, turn);
            dot = row_sum<NT>(dot, lds, turn);
        }
        inv = 1.0f / sqrtf(sum * a.inv_width + a.eps);
        mean = dot * inv * a.inv_width;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
            if (left <= 0) continue;
            float t[8], g[8], o[8];
            load8<FULL>(w + c0, left, t);
            if (x && gain) load8<FULL>(gain + c0, left, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float hn = v[i][e] * inv;
                sw[i][e] += d[i][e] * hn;
                o[e] = (float)h8[i][e] + inv * (d[i][e] * t[e] - hn * mean);
                if (x) sg[i][e] += o[e] * xs[i][e];
            }
            store8<FULL>(gr + base + c0, left, o);
            if (x && gx) {
                if (gain) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] *= g[e];
                }
                store8<FULL>(gx + base + c0, left, o);
            }
        }
    }
    float *out = part + (int64_t)blockIdx.x * 2 * a.width;
    leave_sums<NT, NV>(sw, out, a.width, lds);
    leave_sums<NT, NV>(sg, out + a.width, a.width, lds);
}

struct GateArgs {
    int64_t rows;                                     // tokens * heads
    int heads, width;
    int64_t ldx, ldz, ldy, ldgx, ldgz;                // elements from one token to the next
    float eps, inv_width;
};

// A row's first element: its token's row, and its head in it
__device__ __forceinline__ int64_t gate_at(int64_t token, int head, int64_t ld, int width) { return token * ld + (int64_t)head * width; }

template <class E, int NT, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void norm_gate_kernel(const E *__restrict__ x, const E *__restrict__ z, const float *__restrict__ w,
                                                             E *__restrict__ y, GateArgs a)
{
    __shared__ float lds[8];
    int turn = 0;
    const int lane = threadIdx.x % NT;
    const int64_t row = (int64_t)group_of() * (kThreads / NT) + threadIdx.x / NT;
    const bool live = row < a.rows;
    const int64_t token = live ? row / a.heads : 0;
    const int head = live ? (int)(row - token * a.heads) : 0;
    const E *xp = x + gate_at(token, head, a.ldx, a.width), *zp = z + gate_at(token, head, a.ldz, a.width);
    E *yp = y + gate_at(token, head, a.ldy, a.width);
    float v[NV][8], g[NV][8], sum = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
        if (FULL && left <= 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = g[i][e] = 0;
            continue;
        }
        load8<FULL>(xp + c0, left, v[i]);
        load8<FULL>(zp + c0, left, g[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[i][e] * v[i][e];
    }
    const float inv = 1.0f / sqrtf(row_sum<NT>(sum, lds, turn) * a.inv_width + a.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
        if (left <= 0) continue;
        float t[8];
        load8<FULL>(w + c0, left, t);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= v[i][e] * inv * g[i][e] * sigmoid<E>(g[i][e]);
        store8<FULL>(yp + c0, left, t);
    }
}

template <class E, int NT, int NV, bool FULL>
__global__ __launch_bounds__(kThreads) void norm_gate_grad_kernel(const E *__restrict__ x, const E *__restrict__ z, const float *__restrict__ w,
                                                                  const E *__restrict__ gy, E *__restrict__ gx, E *__restrict__ gz,
                                                                  float *__restrict__ part, GateArgs a)
{
    __shared__ float lds[NT == kThreads ? 16 : 8 * kThreads];
    int turn = 0;
    constexpr int GROUPS = kThreads / NT;
    const int lane = threadIdx.x % NT;
    float sw[NV][8] = {};
    typename Vec<E>::v8 nx[NV], nz[NV], ng[NV];       // the next row, in flight during this one
    auto fetch = [&](int64_t row) {
        const bool live = row < a.rows;
        const int64_t token = live ? row / a.heads : 0;
        const int head = live ? (int)(row - token * a.heads) : 0;
        const E *xp = x + gate_at(token, head, a.ldx, a.width), *zp = z + gate_at(token, head, a.ldz, a.width), *gp = gy + gate_at(token, head, a.ldy, a.width);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
            nx[i] = nz[i] = ng[i] = typename Vec<E>::v8{};
            if (left <= 0) continue;
            nx[i] = fetch8<FULL>(xp + c0, left);
            nz[i] = fetch8<FULL>(zp + c0, left);
            ng[i] = fetch8<FULL>(gp + c0, left);
        }
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    fetch((int64_t)blockIdx.x * GROUPS + threadIdx.x / NT);
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < a.rows; first += step) {
        const int64_t row = first + threadIdx.x / NT;
        const bool live = row < a.rows;
        const int64_t token = live ? row / a.heads : 0;
        const int head = live ? (int)(row - token * a.heads) : 0;
        E *gxp = gx + gate_at(token, head, a.ldgx, a.width), *gzp = gz + gate_at(token, head, a.ldgz, a.width);
        float v[NV][8], zz[NV][8], d[NV][8], sum = 0, dot = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = (float)nx[i][e], zz[i][e] = (float)nz[i][e], d[i][e] = (float)ng[i][e];
            if (left <= 0) continue;                  // (zeros)
            float t[8];
            load8<FULL>(w + c0, left, t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum += v[i][e] * v[i][e];
                dot += d[i][e] * t[e] * (zz[i][e] * sigmoid<E>(zz[i][e])) * v[i][e];
            }
        }
        fetch(row + step);
        sum = row_sum<NT>(sum, lds, turn);
        dot = row_sum<NT>(dot, lds, turn);
        const float inv = 1.0f / sqrtf(sum * a.inv_width + a.eps), mean = dot * inv * a.inv_width;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c0 = (i * NT + lane) * 8, left = live ? a.width - c0 : 0;
            if (left <= 0) continue;
            float t[8], ox[8], oz[8];
            load8<FULL>(w + c0, left, t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = sigmoid<E>(zz[i][e]), act = zz[i][e] * s, xn = v[i][e] * inv;
                sw[i][e] += d[i][e] * act * xn;
                ox[e] = inv * (d[i][e] * act * t[e] - xn * mean);
                oz[e] = d[i][e] * xn * t[e] * (s + act * (1.0f - s));
            }
            store8<FULL>(gxp + c0, left, ox);
            store8<FULL>(gzp + c0, left, oz);
        }
    }
    leave_sums<NT, NV>(sw, part + (int64_t)blockIdx.x * a.width, a.width, lds);
}

// 32 columns x 32 threads of each, then the 32 sums of a column in order of their threads.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *__restrict__ part, float *__restrict__ out, float *__restrict__ more, int64_t split,
                                                           int parts, int64_t stride, int64_t columns)
{
    __shared__ float lds[32][33];
    const int c = threadIdx.x % 32, g = threadIdx.x / 32;
    const int64_t column = (int64_t)group_of() * 32 + c;
    float s = 0;
    if (column < columns) {
        int p = g;
        for (; p + 96 < parts; p += 128) {            // four loads in flight
            const float t0 = part[p * stride + column], t1 = part[(p + 32) * stride + column];
            const float t2 = part[(p + 64) * stride + column], t3 = part[(p + 96) * stride + column];
            s += (t0 + t1) + (t2 + t3);
        }
        for (; p < parts; p += 32) s += part[p * stride + column];
    }
    lds[g][c] = s;
    __syncthreads();
    if (g == 0 && column < columns) {
        s = 0;
        for (int i = 0; i < 32; ++i) s += lds[i][c];
        if (column < split) out[column] = s;
        else if (more) more[column - split] = s;
    }
}

// f<NT, NV>() for rows of `width` columns
template <class F>
hipError_t by_width(int width, F &&f)
{
    if (width <= 64) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    if (width <= 128) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (width <= 256) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    if (width <= 512) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (width <= 1024) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (width <= 2048) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    if (width <= 4096) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    if (width <= 8192) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    return f(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
}

int row_lanes(int width)
{
    return width <= 64 ? 8 : width <= 128 ? 16 : width <= 256 ? 32 : width <= 1024 ? 64 : 256;
}

// Two workgroups per CU have enough loads in flight, and leave few partial rows; eight where those are short.
int grad_groups(int64_t rows, int width)
{
    const int64_t units = (rows * row_lanes(width) + kThreads - 1) / kThreads;
    const int64_t most = (width <= 256 ? 8 : 2) * device_cus();
    return (int)(units < most ? units : most);
}

}  // namespace

hipError_t launch_column_sums(const float *part, float *out, float *more, int64_t split, int parts, int64_t stride, int64_t columns, hipStream_t s)
{
    dim3 grid;
    if (!spread((columns + 31) / 32, 1024, grid)) return kNotTaken;
    hipLaunchKernelGGL(column_sums_kernel, grid, dim3(1024), 0, s, part, out, more, split, parts, stride, columns);
    return hipGetLastError();
}

int64_t norm_add_grad_bytes(int64_t rows, int width) { return 8 * (int64_t)grad_groups(rows, width) * width; }
int64_t norm_gate_grad_bytes(int64_t rows, int width) { return 4 * (int64_t)grad_groups(rows, width) * width; }

hipError_t launch_norm_add(int dtype, const void *r, const void *x, const float *gain, const float *w, void *h, void *n, int64_t rows, int width,
                           float eps, hipStream_t s)
{
    const NormArgs a{rows, width, eps, 1.0f / (float)width};
    const bool full = width % 8 == 0 && sixteen({r, x, gain, w, h, n});
    return by_type(dtype, [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        return by_width(width, [&](auto nt, auto nv) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
            dim3 grid;
            if (!spread((rows + kThreads / NT - 1) / (kThreads / NT), kThreads, grid)) return kNotTaken;
            auto *k = full ? norm_add_kernel<E, NT, NV, true> : norm_add_kernel<E, NT, NV, false>;
            hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, s, (const E *)r, (const E *)x, gain, w, (E *)h, (E *)n, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_norm_add_grad(int dtype, const void *r, const void *x, const float *gain, const float *w, const void *gn, const void *gh, void *gr,
                                void *gx, float *gw, float *ggain, int64_t rows, int width, float eps, Workspace ws, hipStream_t s)
{
    const NormArgs a{rows, width, eps, 1.0f / (float)width};
    const bool full = width % 8 == 0 && sixteen({r, x, gain, w, gn, gh, gr, gx});
    const int groups = grad_groups(rows, width);
    float *part = (float *)ws.p;
    hipError_t e = groups == 0 ? hipSuccess : by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        return by_width(width, [&](auto nt, auto nv) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
            auto *k = full ? norm_add_grad_kernel<E, NT, NV, true> : norm_add_grad_kernel<E, NT, NV, false>;
            hipLaunchKernelGGL(k, dim3(groups), dim3(kThreads), 0, s, (const E *)r, (const E *)x, gain, w, (const E *)gn, (const E *)gh, (E *)gr,
                               (E *)gx, part, a);
            return hipGetLastError();
        });
    });
    if (e == hipSuccess) e = launch_column_sums(part, gw, ggain, width, groups, 2 * (int64_t)width, ggain ? 2 * (int64_t)width : width, s);
    return e;
}

hipError_t launch_norm_gate(int dtype, const void *x, const void *z, const float *w, void *y, int64_t tokens, int heads, int width, int64_t ldx,
                            int64_t ldz, int64_t ldy, float eps, hipStream_t s)
{
    const GateArgs a{tokens * heads, heads, width, ldx, ldz, ldy, 0, 0, eps, 1.0f / (float)width};
    const bool full = width % 8 == 0 && ldx % 8 == 0 && ldz % 8 == 0 && ldy % 8 == 0 && sixteen({x, z, w, y});
    return by_type(dtype, [&](auto *e) {
        using E = std::remove_pointer_t<decltype(e)>;
        return by_width(width, [&](auto nt, auto nv) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
            dim3 grid;
            if (!spread((a.rows + kThreads / NT - 1) / (kThreads / NT), kThreads, grid)) return kNotTaken;
            auto *k = full ? norm_gate_kernel<E, NT, NV, true> : norm_gate_kernel<E, NT, NV, false>;
            hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, s, (const E *)x, (const E *)z, w, (E *)y, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_norm_gate_grad(int dtype, const void *x, const void *z, const float *w, const void *gy, void *gx, void *gz, float *gw,
                                 int64_t tokens, int heads, int width, int64_t ldx, int64_t ldz, int64_t ldgy, int64_t ldgx, int64_t ldgz, float eps,
                                 Workspace ws, hipStream_t s)
{
    const GateArgs a{tokens * heads, heads, width, ldx, ldz, ldgy, ldgx, ldgz, eps, 1.0f / (float)width};
    const bool full = width % 8 == 0 && ldx % 8 == 0 && ldz % 8 == 0 && ldgy % 8 == 0 && ldgx % 8 == 0 && ldgz % 8 == 0 &&
                      sixteen({x, z, w, gy, gx, gz});
    const int groups = grad_groups(a.rows, width);
    float *part = (float *)ws.p;
    hipError_t e = groups == 0 ? hipSuccess : by_type(dtype, [&](auto *t) {
        using E = std::remove_pointer_t<decltype(t)>;
        return by_width(width, [&](auto nt, auto nv) {
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
            auto *k = full ? norm_gate_grad_kernel<E, NT, NV, true> : norm_gate_grad_kernel<E, NT, NV, false>;
            hipLaunchKernelGGL(k, dim3(groups), dim3(kThreads), 0, s, (const E *)x, (const E *)z, w, (const E *)gy, (E *)gx, (E *)gz, part, a);
            return hipGetLastError();
        });
    });
    if (e == hipSuccess) e = launch_column_sums(part, gw, nullptr, width, groups, width, width, s);
    return e;
}

}  // namespace sws

// The gated delta rule over whole sequences: which kernels a call takes, and its workspace.
#include "delta.h"

namespace sws {

hipError_t launch_delta_step(int dtype, int gate_dtype, const void *q, const void *k, const void *v, const void *g, const void *beta, void *o,
                             float *pool, const DeltaArgs &a, hipStream_t s);
hipError_t launch_delta_prep(int dtype, int gate_dtype, const void *q, const void *k, const void *g, const void *beta, char *tri, float *factors,
                             const Magnitudes &mg, int chunks, bool full, bool grad, const DeltaArgs &a, hipStream_t s);
hipError_t launch_delta_scan_16(int dtype, int mode, const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws,
                                const DeltaArgs &a, hipStream_t s);
hipError_t launch_delta_scan_f32(int mode, const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws, const DeltaArgs &a,
                                 hipStream_t s);
hipError_t launch_delta_grad(int dtype, int gate_dtype, const void *q, const void *k, const void *v, const void *g, const void *beta, const void *go, void *gq,
                             void *gk, void *gv, void *gg, void *gbeta, const void *u, const void *r, const void *st, const void *ds, const float *scales,
                             int chunks, int cols, bool full, const DeltaArgs &a, const Steps (&gs)[3], hipStream_t s);

namespace {

int64_t tri_size(int dtype)
{
    return dtype == SWS_DTYPE_F32 ? tri_bytes<float>() : dtype == SWS_DTYPE_BF16 ? tri_bytes<__bf16>() : tri_bytes<_Float16>();
}

int64_t tops_size(int dtype) { return dtype == SWS_DTYPE_F16 ? 8 : 0; }

// Few tokens: one after the other reads and writes the state once and needs no chunk, but takes as much time for every token, and a chunk takes as long
// with one token as with 64.  How many are few depends on what a token costs: with few states a chain of LDS and barriers, with many the
// arithmetic on all of them.  Bf16, states of 128 x 128, one after the other against chunks: 16 states, 8 tokens 11.4 us against 15.5, 12 tokens 15.9 against
// 15.5; 256 states, 12 tokens 29.0 against 36.3, 16 tokens 36.5 against 36.3; 2048 states, 48 tokens 255 against 278, 64 tokens 336 against 288.
bool few(const DeltaArgs &a)
{
    const int64_t states = a.B * a.Hv, cus = device_cus();
    return a.T <= (states < cus ? 8 : states < 8 * cus ? 15 : 48);
}

hipError_t launch_scan(int dtype, int mode, const void *q, const void *k, const void *v, void *o, float *state, const ScanWs &ws, const DeltaArgs &a,
                       hipStream_t s)
{
    return dtype == SWS_DTYPE_F32 ? launch_delta_scan_f32(mode, q, k, v, o, state, ws, a, s) : launch_delta_scan_16(dtype, mode, q, k, v, o, state, ws, a, s);
}

bool full_keys(int dtype, const DeltaArgs &a, const void *q, const void *k)
{
    if (a.Dk != 64 && a.Dk != 128) return false;
    if (dtype == SWS_DTYPE_F32) return full_rows<float>(a.q, a.Dk, q) && full_rows<float>(a.k, a.Dk, k);
    return full_rows<__bf16>(a.q, a.Dk, q) && full_rows<__bf16>(a.k, a.Dk, k);
}

// (whole blocks of 32 columns)
bool full_grads(int dtype, const DeltaArgs &a, const void *v, const void *go, const void *gq, const void *gk, const void *gv, const Steps (&gs)[3])
{
    if (a.Dv % 32) return false;
    if (dtype == SWS_DTYPE_F32)
        return full_rows<float>(a.v, 32, v) && full_rows<float>(a.o, 32, go) && full_rows<float>(gs[0], a.Dk, gq) && full_rows<float>(gs[1], a.Dk, gk) &&
               full_rows<float>(gs[2], 32, gv);
    return full_rows<__bf16>(a.v, 32, v) && full_rows<__bf16>(a.o, 32, go) && full_rows<__bf16>(gs[0], a.Dk, gq) && full_rows<__bf16>(gs[1], a.Dk, gk) &&
           full_rows<__bf16>(gs[2], 32, gv);
}

int keys(const DeltaArgs &a) { return a.Dk <= 64 ? 64 : 128; }
int columns(const DeltaArgs &a) { return (a.Dv + 31) / 32 * 32; }

}  // namespace

int64_t delta_rule_bytes(int dtype, const DeltaArgs &a)
{
    if (few(a)) return 0;
    return a.B * a.Hv * ((a.T + kChunk - 1) / kChunk) * (2 * tri_size(dtype) + kFactorBytes + tops_size(dtype));
}

// T, T^T and P^T; the chunks' factors; U and dR; the states before the chunks and the gradients of those behind them; magnitudes and the heads' scales
int64_t delta_rule_grad_bytes(int dtype, const DeltaArgs &a)
{
    const int64_t n = a.B * a.Hv * ((a.T + kChunk - 1) / kChunk);
    return n * (3 * tri_size(dtype) + kFactorBytes + 8 * (int64_t)(kChunk + keys(a)) * columns(a) + tops_size(dtype)) + a.B * a.Hv * tops_size(dtype);
}

hipError_t launch_delta_rule(int dtype, int gate_dtype, const void *q, const void *k, const void *v, const void *g, const void *beta, void *o,
                             float *pool, const DeltaArgs &a, Workspace ws, hipStream_t s)
{
    if (few(a)) return launch_delta_step(dtype, gate_dtype, q, k, v, g, beta, o, pool, a, s);
    const int64_t chunks = (a.T + kChunk - 1) / kChunk;
    if (chunks > 0x7fffff) return kNotTaken;
    char *tri = (char *)ws.p;
    const int64_t n = a.B * a.Hv * chunks;
    float *factors = (float *)(tri + n * 2 * tri_size(dtype));
    unsigned *tops = (unsigned *)((char *)factors + n * kFactorBytes);
    hipError_t e = launch_delta_prep(dtype, gate_dtype, q, k, g, beta, tri, factors, {v, nullptr, pool, nullptr, tops}, (int)chunks, full_keys(dtype, a, q, k), false,
                                     a, s);
    if (e == hipSuccess) e = launch_scan(dtype, FORWARD, q, k, v, o, pool, {tri, factors, nullptr, nullptr, tops, nullptr, (int)chunks, 0}, a, s);
    return e;
}

hipError_t launch_delta_rule_grad(int dtype, int gate_dtype, const void *q, const void *k, const void *v, const void *g, const void *beta, const void *go,
                                  const float *state, float *gstate, void *gq, void *gk, void *gv, void *gg, void *gbeta, const DeltaArgs &a,
                                  const Steps (&gs)[3], Workspace ws, hipStream_t s)
{
    const int64_t chunks = (a.T + kChunk - 1) / kChunk, n = a.B * a.Hv * chunks;
    if (chunks > 0x7fffff) return kNotTaken;
    const int cols = columns(a), nc = (int)chunks;
    char *tri = (char *)ws.p;
    float *factors = (float *)(tri + n * 3 * tri_size(dtype));
    float *u = factors + n * (kFactorBytes / 4), *r = u + n * kChunk * cols, *st = r + n * kChunk * cols, *ds = st + n * keys(a) * cols;
    unsigned *tops = (unsigned *)(ds + n * keys(a) * cols);
    float *scales = (float *)(tops + 2 * n);
    const bool fk = full_keys(dtype, a, q, k);
    hipError_t e = launch_delta_prep(dtype, gate_dtype, q, k, g, beta, tri, factors, {v, go, state, gstate, tops}, nc, fk, true, a, s);
    if (e == hipSuccess) e = launch_scan(dtype, KEEP, q, k, v, nullptr, const_cast<float *>(state), {tri, factors, u, st, tops, scales, nc, cols}, a, s);
    if (e == hipSuccess) e = launch_scan(dtype, BACKWARD, q, k, v, const_cast<void *>(go), gstate, {tri, factors, r, ds, tops, scales, nc, cols}, a, s);
    const bool full = fk && full_grads(dtype, a, v, go, gq, gk, gv, gs);
    if (e == hipSuccess)
        e = launch_delta_grad(dtype, gate_dtype, q, k, v, g, beta, go, gq, gk, gv, gg, gbeta, u, r, st, ds, scales, nc, cols, full, a, gs, s);
    return e;
}

}  // namespace sws

// The weighted sum of the experts' rows of a token, and its gradient.
//
// Bound by memory: forward every row of Y passes once; backward it passes once for the weights' gradient, beside a pass over dout for every four rows (from memory
// one, the others from the cache), and every row of dY goes out once, the padding among them cleared by workgroups of their own.  No atomics: a token's
// waves hold all that its gradients need.  8191 tokens of 4 rows of 4096 in bf16: 61 us forward (335 MB, 5.5 TB/s), 119 back (608 MB, 5.1 TB/s);
// 4095 of 8 rows 56 and 109 (5.2 TB/s back); a large copy reaches 4.7.
#include "experts_common.hpp"

using namespace hgemm;

namespace {

constexpr int kMostChoices = 32;

struct CombineArgs {
    const int* rows;
    const int* tokens_of;
    const float* weights;
    const void* Y;
    void* out;              // backward: dout
    void* dY;
    float* dweights;
    int64_t ldy, ldo, tokens, y_rows;
    int N, k;
    int wide;               // all rows start on 16 bytes and hold whole groups of eight
};

template <class T> __device__ __forceinline__ Eight<T> load_eight(const void* base, int64_t row, int64_t ld, int n, int N, bool wide)
{
    Eight<T> x{};
    x.load((const T*)base + row * ld + n, N - n, wide);
    return x;
}

// A wave takes 512 columns of a token: 8 columns a lane.
constexpr int kWaveCols = 512;
template <class Y, class O> __global__ __launch_bounds__(256) void combine_kernel(CombineArgs a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int parts = (a.N + kWaveCols - 1) / kWaveCols;
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave;
    const int64_t t = unit / parts;
    const int n = (int)(unit - t * parts) * kWaveCols + lane * 8;
    if (t >= a.tokens || n >= a.N) return;
    float sum[8] = {};
    for (int j0 = 0; j0 < a.k; j0 += 4) {               // four rows in flight
        Eight<Y> y[4];
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = j0 + j < a.k ? a.rows[t * a.k + j0 + j] : -1;
            y[j] = Eight<Y>{};
            w[j] = 0.f;
            if ((uint64_t)(int64_t)r >= (uint64_t)a.y_rows) continue;
            w[j] = a.weights ? a.weights[t * a.k + j0 + j] : 1.f;
            y[j] = load_eight<Y>(a.Y, r, a.ldy, n, a.N, a.wide);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += w[j] * y[j].value(e);
    }
    Eight<O> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o.set(e, from_float<O>(sum[e]));
    o.store((O*)a.out + t * a.ldo + n, a.N - n, a.wide);
}

// WPT waves take a token, all columns of it: dout passes once for every four of the token's rows of Y and dY.  The workgroups behind those of the tokens
// look through 64 rows of dY each and clear the padding among them.
template <class Y, class O, int WPT> __global__ __launch_bounds__(256) void combine_backward_kernel(CombineArgs a)
{
    constexpr int TOKENS = 4 / WPT;
    const int64_t of_tokens = (a.tokens + TOKENS - 1) / TOKENS;
    if ((int64_t)blockIdx.x >= of_tokens) {
        const int64_t r0 = ((int64_t)blockIdx.x - of_tokens) * 64;
        const int64_t mine = r0 + (threadIdx.x & 63);
        const uint64_t clear = __ballot(mine < a.y_rows && a.tokens_of[mine < a.y_rows ? mine : 0] < 0);
        int per = 8;                                    // threads side by side on a row
        while (per < 256 && per * 8 < a.N) per *= 2;
        const Eight<Y> zero{};
        for (int i = threadIdx.x / per; i < 64; i += 256 / per) {
            if (!(clear >> i & 1)) continue;
            for (int n = threadIdx.x % per * 8; n < a.N; n += per * 8) zero.store((Y*)a.dY + (r0 + i) * a.ldy + n, a.N - n, a.wide);
        }
        return;
    }
    __shared__ float part[4][4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + wave / WPT;
    if (WPT == 1 && t >= a.tokens) return;
    for (int j0 = 0; j0 < a.k; j0 += 4) {               // four rows at a time
        int r[4];
        float w[4], dot[4] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            r[j] = j0 + j < a.k ? a.rows[t * a.k + j0 + j] : -1;
            if ((uint64_t)(int64_t)r[j] >= (uint64_t)a.y_rows) r[j] = -1;
            w[j] = r[j] >= 0 && a.weights ? a.weights[t * a.k + j0 + j] : 1.f;
        }
        for (int n = (wave % WPT) * kWaveCols + lane * 8; n < a.N; n += WPT * kWaveCols) {
            const Eight<O> d = load_eight<O>(a.out, t, a.ldo, n, a.N, a.wide);
            if (a.dweights) {
                Eight<Y> y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    y[j] = Eight<Y>{};
                    if (r[j] >= 0) y[j] = load_eight<Y>(a.Y, r[j], a.ldy, n, a.N, a.wide);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot[j] += d.value(e) * y[j].value(e);
            }
            if (a.dY) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (r[j] < 0) continue;
                    Eight<Y> o;
#pragma unroll
                    for (int e = 0; e < 8; ++e) o.set(e, from_float<Y>(w[j] * d.value(e)));
                    o.store((Y*)a.dY + r[j] * a.ldy + n, a.N - n, a.wide);
                }
            }
        }
        if (!a.dweights) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (r[j] < 0) dot[j] = 0.f;                 // also beside an infinite dout
#pragma unroll
            for (int s = 1; s < 64; s *= 2) dot[j] += __shfl_xor(dot[j], s);
        }
        if constexpr (WPT == 1) {
            if (lane < 4 && j0 + lane < a.k) a.dweights[t * a.k + j0 + lane] = lane == 0 ? dot[0] : lane == 1 ? dot[1] : lane == 2 ? dot[2] : dot[3];
        } else {
            if (lane == 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) part[wave][j] = dot[j];
            }
            __syncthreads();
            if (threadIdx.x < 4 && j0 + (int)threadIdx.x < a.k)
                a.dweights[t * a.k + j0 + threadIdx.x] = part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x];
            __syncthreads();
        }
    }
}

int64_t workgroups(const CombineArgs& a, bool backward)
{
    if (!backward) return (a.tokens * ((a.N + (int64_t)kWaveCols - 1) / kWaveCols) + 3) / 4;
    return (a.N <= kWaveCols ? (a.tokens + 3) / 4 : a.tokens) + (a.dY ? (a.y_rows + 63) / 64 : 0);
}

template <class Y, class O> void launch(const CombineArgs& a, bool backward, hipStream_t s)
{
    const unsigned grid = (unsigned)workgroups(a, backward);
    if (!grid) return;
    if (!backward) combine_kernel<Y, O><<<grid, 256, 0, s>>>(a);
    else if (a.N <= kWaveCols) combine_backward_kernel<Y, O, 1><<<grid, 256, 0, s>>>(a);
    else combine_backward_kernel<Y, O, 4><<<grid, 256, 0, s>>>(a);
}

template <class Y> void launch_out(const CombineArgs& a, hgemm_type_t out, bool backward, hipStream_t s)
{
    if (out == HGEMM_F16) launch<Y, _Float16>(a, backward, s);
    else if (out == HGEMM_BF16) launch<Y, __bf16>(a, backward, s);
    else launch<Y, float>(a, backward, s);
}

// Checks what both directions share.
hgemm_status_t start(const hgemm_combine_t* d, CombineArgs& a, const int32_t* rows, const void* Y, const void* out)
{
    if (!d || (unsigned)d->y > HGEMM_F32 || (unsigned)d->out > HGEMM_F32 || d->tokens < 0 || d->N < 0 || d->y_rows < 0 || d->k < 1 || d->k > kMostChoices) return HGEMM_ERR_INVALID_ARG;
    a = CombineArgs{};
    a.ldy = d->ldy ? d->ldy : d->N;
    a.ldo = d->ldo ? d->ldo : d->N;
    if (a.ldy < d->N || a.ldo < d->N) return HGEMM_ERR_INVALID_ARG;
    if (d->N > 0x7fffff00LL || d->tokens > 0x7fffff00LL || d->y_rows > 0x7fffff00LL) return HGEMM_ERR_UNSUPPORTED;
    a.tokens = d->tokens; a.y_rows = d->y_rows; a.N = (int)d->N; a.k = d->k;
    if (!aligned(rows, 4) || !aligned(Y, type_size(d->y)) || !aligned(out, type_size(d->out))) return HGEMM_ERR_INVALID_ARG;
    return HGEMM_OK;
}

hgemm_status_t go(const hgemm_combine_t* d, CombineArgs& a, bool backward, void* hip_stream)
{
    if (!fits_grid(workgroups(a, backward), 256)) return HGEMM_ERR_UNSUPPORTED;
    if (!current_device_is_gfx950()) return HGEMM_ERR_ARCH;
    a.wide = a.N % 8 == 0 && a.ldy * type_size(d->y) % 16 == 0 && a.ldo * type_size(d->out) % 16 == 0 && aligned(a.Y, 16) && aligned(a.out, 16) && aligned(a.dY, 16);
    const hipStream_t s = (hipStream_t)hip_stream;
    if (d->y == HGEMM_F16) launch_out<_Float16>(a, d->out, backward, s);
    else if (d->y == HGEMM_BF16) launch_out<__bf16>(a, d->out, backward, s);
    else launch_out<float>(a, d->out, backward, s);
    return hipGetLastError() == hipSuccess ? HGEMM_OK : HGEMM_ERR_LAUNCH;
}

}  // namespace

extern "C" hgemm_status_t hgemm_combine(const hgemm_combine_t* d, const int32_t* rows, const float* weights, const void* Y, void* out, void* hip_stream)
{
    CombineArgs a;
    const hgemm_status_t st = start(d, a, rows, Y, out);
    if (st != HGEMM_OK) return st;
    if (!d->tokens || !d->N) return HGEMM_OK;
    if (!rows || !out || (d->y_rows && !Y) || !aligned(weights, 4)) return HGEMM_ERR_INVALID_ARG;
    a.rows = rows; a.weights = weights; a.Y = Y; a.out = out;
    return go(d, a, false, hip_stream);
}

extern "C" hgemm_status_t hgemm_combine_backward(const hgemm_combine_t* d, const int32_t* rows, const int32_t* tokens_of, const float* weights, const void* Y, const void* dout, void* dY,
                                                 float* dweights, void* hip_stream)
{
    CombineArgs a;
    const hgemm_status_t st = start(d, a, rows, Y, dout);
    if (st != HGEMM_OK) return st;
    if ((!d->tokens && !d->y_rows) || (!dY && !dweights)) return HGEMM_OK;
    if ((d->tokens && (!rows || (d->N && !dout))) || (dweights && d->y_rows && !Y) || (dY && d->y_rows && !tokens_of)) return HGEMM_ERR_INVALID_ARG;
    if (!aligned(weights, 4) || !aligned(dweights, 4) || !aligned(tokens_of, 4) || !aligned(dY, type_size(d->y))) return HGEMM_ERR_INVALID_ARG;
    a.rows = rows; a.tokens_of = tokens_of; a.weights = weights; a.Y = Y; a.out = (void*)dout; a.dY = dY; a.dweights = dweights;
    return go(d, a, true, hip_stream);
}

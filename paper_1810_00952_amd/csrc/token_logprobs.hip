// Log probabilities of given tokens, with entropy and the largest logits of a row, and the gradient:
//
//   m = max x,  S = sum e^(x - m),  U = sum (x - m) e^(x - m)
//   lp = x[tok] - m - ln S,   ent = ln S - U / S,   dx = dlp (1[v = tok] - p) - dent p (ln p + ent)
//
// A row of -inf alone: lp -inf, ent 0, dx 0.  A row with +inf or NaN: NaN.
#include "device_utils.h"

namespace rl {

namespace {

constexpr int WG = 256;

// maximum, S and U of x - m; a term of -inf adds nothing to either
struct Soft { float m, s, u; };

__device__ __forceinline__ Soft join(const Soft &a, const Soft &b)
{
    Soft r;
    r.m = fmaxf(a.m, b.m);
    // a side that has seen nothing above -inf has s = u = 0
    const float da = a.m == -INFINITY ? 0.0f : a.m - r.m, db = b.m == -INFINITY ? 0.0f : b.m - r.m;
    const float ea = __expf(da), eb = __expf(db);
    r.s = a.s * ea + b.s * eb;
    r.u = (a.u + a.s * da) * ea + (b.u + b.s * db) * eb;
    return r;
}

// the order of the alternatives as one number: larger for the larger logit, then for the earlier one; NaN above everything
__device__ __forceinline__ uint64_t rank_key(float x, int64_t v)
{
    uint32_t u = __float_as_uint(x + 0.0f);
    u = x != x ? 0xfffffffeu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return ((uint64_t)u << 32) | (0xffffffffu - (uint32_t)v);
}

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int o)
{
    return ((uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), o) << 32) | (uint32_t)__shfl_xor((int)(uint32_t)v, o);
}

// statistics of the row, in every thread
__device__ __forceinline__ Soft row_stats(const void *x, int dtype, int64_t at, int64_t V)
{
    float m = -INFINITY;
    for (int64_t v = threadIdx.x; v < V; v += WG) {
        const float f = load_as_f32(x, dtype, at + v);
        m = f != f ? INFINITY : fmaxf(m, f);
    }
    Soft a{m, 0.0f, 0.0f};
    if (m > -INFINITY)
        for (int64_t v = threadIdx.x; v < V; v += WG) {
            const float f = load_as_f32(x, dtype, at + v);
            if (f != -INFINITY) {
                const float d = f - m, e = __expf(d);
                a.s += e; a.u += d * e;
            }
        }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) a = join(a, Soft{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.u, o)});
    __shared__ Soft sh[WG / 64];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = a;
    __syncthreads();
    a = sh[0];
#pragma unroll
    for (int i = 1; i < WG / 64; ++i) a = join(a, sh[i]);
    return a;
}

}  // namespace

__global__ __launch_bounds__(WG) void token_logprobs_kernel(const LogprobsParams p)
{
    const int64_t row = blockIdx.x, at = row * p.V;
    const Soft a = row_stats(p.x, p.dtype, at, p.V);
    const bool dead = a.m == -INFINITY, broken = a.m == INFINITY;
    const float ls = logf(a.s);
    auto logp = [&](float x) { return broken ? __builtin_nanf("") : dead ? -INFINITY : x - a.m - ls; };
    if (threadIdx.x == 0) {
        const int tok = p.tok[row];
        const bool given = tok >= 0 && tok < p.V;
        p.lp[row] = broken ? __builtin_nanf("") : given ? logp(load_as_f32(p.x, p.dtype, at + tok)) : 0.0f;
        p.ent[row] = broken ? __builtin_nanf("") : dead ? 0.0f : ls - a.u / a.s;
    }
    __shared__ uint64_t sh[WG / 64];
    uint64_t last = ~(uint64_t)0;
    for (int k = 0; k < p.top; ++k) {
        uint64_t best = 0;                                  // below every key: an index is under 2^31
        for (int64_t v = threadIdx.x; v < p.V; v += WG) {
            const uint64_t key = rank_key(load_as_f32(p.x, p.dtype, at + v), v);
            if (key < last && key > best) best = key;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { const uint64_t other = shfl_xor64(best, o); best = other > best ? other : best; }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = best;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WG / 64; ++i) best = sh[i] > best ? sh[i] : best;
        last = best;
        if (threadIdx.x == 0) {
            const uint32_t id = 0xffffffffu - (uint32_t)best;
            p.top_id[row * p.top + k] = (int32_t)id;
            p.top_lp[row * p.top + k] = logp(load_as_f32(p.x, p.dtype, at + id));
        }
    }
}

__global__ __launch_bounds__(WG) void token_logprobs_grad_kernel(const LogprobsParams p)
{
    const int64_t row = blockIdx.x, at = row * p.V;
    const Soft a = row_stats(p.x, p.dtype, at, p.V);
    const bool dead = a.m == -INFINITY, broken = a.m == INFINITY;
    const float ls = logf(a.s), inv = 1.0f / a.s, ent = ls - a.u * inv;
    const int tok = p.tok[row];
    const float dlp = tok >= 0 && tok < p.V ? p.dlp[row] : 0.0f, dent = p.dent[row];
    for (int64_t v = threadIdx.x; v < p.V; v += WG) {
        const float x = load_as_f32(p.x, p.dtype, at + v);
        float dx = v == tok ? dlp : 0.0f;
        if (x != -INFINITY) {
            const float d = x - a.m, pr = __expf(d) * inv;
            dx -= pr * (dlp + dent * (d - ls + ent));
        }
        store_from_f32(p.dx, p.dtype, at + v, broken ? __builtin_nanf("") : dead ? 0.0f : dx);
    }
}

int64_t logprobs_part_floats(const LogprobsParams &, bool) { return 0; }

hipError_t launch_logprobs(const LogprobsParams &p, hipStream_t s)
{
    if (p.M < 1 || p.V < 1 || p.M > 0x7fffffff || p.V > 0x7fffffff || p.top < 0 || p.top > p.V) return hipErrorInvalidValue;
    hipLaunchKernelGGL(token_logprobs_kernel, dim3((unsigned)p.M), dim3(WG), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_logprobs_grad(const LogprobsParams &p, hipStream_t s)
{
    if (p.M < 1 || p.V < 1 || p.M > 0x7fffffff || p.V > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(token_logprobs_grad_kernel, dim3((unsigned)p.M), dim3(WG), 0, s, p);
    return hipGetLastError();
}

}  // namespace rl

// Root-mean-square norm of a residual stream, with the residual's addition, into 8-bit values with a scale per row:
//
//   y = x + r (rounded as it is stored);  i = (mean y^2 + eps)^-1/2;  s = i max|y g| / 127;  q = rint(y g 127 / max|y g|)
//
// i cancels out of q, so the row's sum of squares and its largest |y g| are one reduction.
#include "device_utils.h"

namespace rl {

namespace {

constexpr int WG = 256;

// sum of a and largest of b over the workgroup, in every thread
__device__ __forceinline__ void reduce_sum_max(float &a, float &b)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        a += __shfl_xor(a, o);
        b = fmaxf(b, __shfl_xor(b, o));
    }
    __shared__ float sa[WG / 64], sb[WG / 64];
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) { sa[w] = a; sb[w] = b; }
    __syncthreads();
    a = sa[0]; b = sb[0];
#pragma unroll
    for (int i = 1; i < WG / 64; ++i) { a += sa[i]; b = fmaxf(b, sb[i]); }
}

}  // namespace

__global__ __launch_bounds__(WG) void norm_q8_kernel(const NormQ8Params p)
{
    const int64_t row = blockIdx.x, at = row * p.D;
    float sum = 0.0f, most = 0.0f;
    for (int64_t d = threadIdx.x; d < p.D; d += WG) {
        float y = load_as_f32(p.x, p.dtype, at + d);
        if (p.r) {
            y += load_as_f32(p.r, p.dtype, at + d);
            store_from_f32(p.y, p.dtype, at + d, y);
            if (p.dtype == DT_BF16) y = round_bf16(y);
        }
        sum += y * y;
        most = fmaxf(most, fabsf(y * load_as_f32(p.g, p.g_dtype, d)));
    }
    reduce_sum_max(sum, most);
    // an infinity or NaN in the row is one in its sum of squares
    const bool whole = sum < INFINITY && most < INFINITY;
    const float inv = rsqrtf(sum / (float)p.D + p.eps);
    const float up = most < 1e-30f ? 0x1p100f : 1.0f;              // the factor of a tiny row would be past f32
    const float to_q = whole && most > 0.0f ? 127.0f / (most * up) : 0.0f;
    if (threadIdx.x == 0) p.s[row] = whole ? most * inv / 127.0f : __builtin_nanf("");
    for (int64_t d = threadIdx.x; d < p.D; d += WG) {
        float y = load_as_f32(p.x, p.dtype, at + d);
        if (p.r) {
            y += load_as_f32(p.r, p.dtype, at + d);
            if (p.dtype == DT_BF16) y = round_bf16(y);
        }
        const float n = whole ? y * load_as_f32(p.g, p.g_dtype, d) * up * to_q : 0.0f;
        p.q[at + d] = (int8_t)rintf(fminf(fmaxf(n, -127.0f), 127.0f));
    }
}

hipError_t launch_norm_q8(const NormQ8Params &p, hipStream_t s)
{
    if (p.M < 1 || p.D < 1 || p.M > 0x7fffffff || (p.r != nullptr) != (p.y != nullptr)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(norm_q8_kernel, dim3((unsigned)p.M), dim3(WG), 0, s, p);
    return hipGetLastError();
}

}  // namespace rl

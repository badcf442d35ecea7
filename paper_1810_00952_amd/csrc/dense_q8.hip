// Product of 8-bit integers with a scale per row of x and per row of w:
//
//   y[m, n] = sx[m] sw[n] sum_k x[m, k] w[n, k] + b[n],   the sum exact in 32 bits
#include "device_utils.h"

namespace rl {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// One wave, one 32 x 32 tile: w's rows are the MFMA's rows, so that a lane holds one row of x.  Lane l's sixteen bytes of a fragment
// are k = 16 (l >> 5) .. +15 of row l & 31, the same in both operands.
__global__ __launch_bounds__(64) void dense_q8_kernel(const DenseQ8Params p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int lane = threadIdx.x, r = lane & 31, half = lane >> 5;
    const int64_t tiles_m = (p.M + 31) / 32, m0 = blockIdx.x % tiles_m * 32, n0 = blockIdx.x / tiles_m * 32;
    const int64_t m = m0 + r, n = min(n0 + r, p.N - 1);
    const int8_t *xr = p.x + min(m, p.M - 1) * p.ldx + 16 * half, *wr = p.w + n * p.ldw + 16 * half;
    i32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0;
    // w's row is zero behind K, x's row is read to its own end only
    for (int64_t k = 0; k < p.ldw; k += 32) {
        const i32x4 zero = {0, 0, 0, 0};
        const i32x4 a = *(const i32x4 *)(wr + k), b = k + 16 * half < p.ldx ? *(const i32x4 *)(xr + k) : zero;
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
    if (m >= p.M) return;
    const float sx = p.sx[m];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t col = n0 + (i & 3) + 8 * (i >> 2) + 4 * half;
        if (col < p.N) {
            float v = (float)acc[i] * sx * p.sw[col];
            if (p.b) v += p.b[col];
            store_from_f32(p.y, p.y_dtype, m * p.N + col, v);
        }
    }
#endif
}

hipError_t launch_dense_q8(const DenseQ8Params &p, hipStream_t s)
{
    const int64_t tiles = ((p.M + 31) / 32) * ((p.N + 31) / 32);
    if (p.M < 1 || p.N < 1 || p.K < 1 || p.ldx < p.K || p.ldw < p.K || p.ldx % 16 != 0 || p.ldw % 128 != 0 || tiles > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(dense_q8_kernel, dim3((unsigned)tiles), dim3(64), 0, s, p);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// rows of K bytes into rows of Kp, the bytes behind them zero
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pad_bytes_kernel(const uint8_t *__restrict__ src, uint8_t *__restrict__ dst, const PadBytes p)
{
    const int64_t vecs = p.Kp / 16, total = p.R * vecs;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / vecs, k = (i - r * vecs) * 16;
        const uint8_t *from = src + r * p.K + k;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (k + 16 <= p.K) {
            __builtin_memcpy(&v, from, 16);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (k + j < p.K) v[j >> 2] |= (uint32_t)from[j] << (8 * (j & 3));
        }
        *(u32x4 *)(dst + r * p.Kp + k) = v;
    }
}

hipError_t launch_pad_bytes(const void *src, void *dst, const PadBytes &p, hipStream_t s)
{
    if (p.R < 1 || p.K < 1 || p.Kp < p.K || p.Kp % 16 != 0) return hipErrorInvalidValue;
    const int64_t blocks = (p.R * (p.Kp / 16) + 255) / 256;
    hipLaunchKernelGGL(pad_bytes_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, (const uint8_t *)src, (uint8_t *)dst, p);
    return hipGetLastError();
}

}  // namespace rl

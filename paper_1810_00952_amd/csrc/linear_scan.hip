// Gated linear recurrence over the rows of a sequence, every channel by itself:
//
//   h_t = a_t h_(t-1) + (1 - a_t) v_t,   a_t = sigmoid(f_t),   state in f32
//
// and its gradient, the same recurrence backwards: G_t = dh_t + a_(t+1) G_(t+1),
//   dv_t = G_t (1 - a_t),   df_t = G_t (h_(t-1) - v_t) a_t (1 - a_t).
// keep[t] = 0: padding, which holds the state; 2: the state before it is zero.
#include "device_utils.h"

namespace rl {

namespace {

// sigmoid(f) and 1 - sigmoid(f), each to its own last bits
__device__ __forceinline__ void gate(float f, float &a, float &rest)
{
    a = rcp_(1.0f + __expf(-f));
    rest = rcp_(1.0f + __expf(f));
}

}  // namespace

__global__ __launch_bounds__(64) void linear_scan_kernel(const ScanParams p)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (c >= p.B * p.D) return;
    const int64_t b = c / p.D, d = c - b * p.D;
    float h = p.h0[c];
    for (int64_t t = 0; t < p.T; ++t) {
        const int64_t row = b * p.T + t;
        const int keep = p.keep ? p.keep[row] : 1;
        float out = 0.0f;
        if (keep) {
            float a, rest;
            gate(load_as_f32(p.z, p.dtype, row * 2 * p.D + d), a, rest);
            const float u = rest * load_as_f32(p.z, p.dtype, row * 2 * p.D + p.D + d);
            h = keep == 2 ? u : __builtin_fmaf(a, h, u);
            out = h;
        }
        store_from_f32(p.h, p.dtype, row * p.D + d, out);
    }
    p.hT[c] = h;
}

__global__ __launch_bounds__(64) void linear_scan_grad_kernel(const ScanParams p)
{
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (c >= p.B * p.D) return;
    const int64_t b = c / p.D, d = c - b * p.D;
    float h = p.h0[c];
    for (int64_t t = 0; t < p.T; ++t) {                     // the states between, into the scratch
        const int64_t row = b * p.T + t;
        const int keep = p.keep ? p.keep[row] : 1;
        p.part[row * p.D + d] = keep == 2 ? 0.0f : h;
        if (keep) {
            float a, rest;
            gate(load_as_f32(p.z, p.dtype, row * 2 * p.D + d), a, rest);
            const float u = rest * load_as_f32(p.z, p.dtype, row * 2 * p.D + p.D + d);
            h = keep == 2 ? u : __builtin_fmaf(a, h, u);
        }
    }
    float G = p.dhT[c];
    for (int64_t t = p.T - 1; t >= 0; --t) {
        const int64_t row = b * p.T + t;
        const int keep = p.keep ? p.keep[row] : 1;
        float df = 0.0f, dv = 0.0f;
        if (keep) {
            float a, rest;
            gate(load_as_f32(p.z, p.dtype, row * 2 * p.D + d), a, rest);
            const float v = load_as_f32(p.z, p.dtype, row * 2 * p.D + p.D + d);
            G += load_as_f32(p.dh, p.dtype, row * p.D + d);
            dv = G * rest;
            df = dv * (p.part[row * p.D + d] - v) * a;
            G = keep == 2 ? 0.0f : a * G;
        }
        store_from_f32(p.dz, p.dtype, row * 2 * p.D + d, df);
        store_from_f32(p.dz, p.dtype, row * 2 * p.D + p.D + d, dv);
    }
    p.dh0[c] = G;
}

int64_t scan_part_floats(const ScanParams &p, bool grad) { return grad ? p.B * p.T * p.D : 0; }

static bool sizes_ok(const ScanParams &p) { return p.B >= 1 && p.T >= 1 && p.D >= 1 && (p.B * p.D + 63) / 64 <= 0x7fffffff; }

hipError_t launch_scan(const ScanParams &p, hipStream_t s)
{
    if (!sizes_ok(p)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(linear_scan_kernel, dim3((unsigned)((p.B * p.D + 63) / 64)), dim3(64), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_scan_grad(const ScanParams &p, hipStream_t s)
{
    if (!sizes_ok(p)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(linear_scan_grad_kernel, dim3((unsigned)((p.B * p.D + 63) / 64)), dim3(64), 0, s, p);
    return hipGetLastError();
}

}  // namespace rl

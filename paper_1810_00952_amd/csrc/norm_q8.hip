// Root-mean-square norm of a residual stream, with the residual's addition, into 8-bit values with a scale per row:
//
//   y = x + r (rounded as it is stored);  i = (mean y^2 + eps)^-1/2;  s = i max|y g| / 127;  q = rint(y g 127 / max|y g|)
//
// i cancels out of q, so the row's sum of squares and its largest |y g| are one reduction.  A workgroup holds its row in registers
// and reads it once; what bounds it is HBM: 16384 x 4096 bf16 with the residual 79 us (5.9 TB/s).  Rows past 128 KB are read twice.
#include "row_vectors.h"

namespace rl {

namespace {

// sum of a and largest of b over the workgroup of T threads, in every thread
template <int T>
__device__ __forceinline__ void reduce_sum_max(float &a, float &b)
{
    a = wave_sum(a);
    b = wave_max(b);
    if constexpr (T > 64) {
        __shared__ float sa[T / 64], sb[T / 64];
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        if (lane == 0) { sa[w] = a; sb[w] = b; }
        __syncthreads();
        a = wave_sum(lane < T / 64 ? sa[lane] : 0.0f);
        b = wave_max(lane < T / 64 ? sb[lane] : 0.0f);
    }
}

// the largest of |y g| by their bits, which order NaN above everything; where there is one, the sum of squares says so
struct Largest {
    uint32_t bits = 0;
    __device__ __forceinline__ void take(float yg) { bits = max(bits, __float_as_uint(yg) & 0x7fffffffu); }
    __device__ __forceinline__ float value(float &sum) const
    {
        if (bits > 0x7f800000u) sum = __builtin_nanf("");
        return __uint_as_float(bits);
    }
};

// what becomes of a row: its scale, and the factors that take y g to the number that is rounded
struct Scale {
    float s, up, to_q;
    bool whole;
    __device__ __forceinline__ Scale(const NormQ8Params &p, float sum, float most)
    {
        whole = sum < INFINITY && most < INFINITY;                  // an infinity or NaN in the row or NaN among y g is one in its sum of squares
        const float i = rsqrtf(sum / (float)p.D + p.eps);
        s = most * i / 127.0f;
        if (!(s < INFINITY)) s = most / 127.0f * i;                 // 127 steps may be past f32 where one is not
        whole = whole && s < INFINITY;
        s = whole ? s : __builtin_nanf("");
        up = most < 1e-30f ? 0x1p100f : 1.0f;                       // the factor of a tiny row would be past f32
        to_q = whole && most > 0.0f ? 127.0f / (most * up) : 0.0f;
    }
    __device__ __forceinline__ int quantised(float yg) const
    {
        const float n = whole ? yg * up * to_q : 0.0f;
        return (int)rintf(fminf(fmaxf(n, -127.0f), 127.0f));
    }
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// the gains of columns c .. c + N - 1, all of them there
template <int N> __device__ __forceinline__ void gains(const NormQ8Params &p, int32_t c, float (&g)[N])
{
    if (p.g_dtype == DT_F32) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const f32x4_any v = *(const f32x4_any *)((const float *)p.g + c + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[k + i] = v[i];
        }
    } else if (p.D % N == 0) {
        if constexpr (N == 8) load8(p.g, DT_BF16, c, g);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) g[k] = load_as_f32(p.g, DT_BF16, c + k);
    }
}

}  // namespace

template <typename E, int T, int NV, bool RES>
__global__ __launch_bounds__(T) void norm_q8_row_kernel(const NormQ8Params p)
{
    typedef RowVectors<E, T, NV> Row;
    constexpr int N = Row::N;
    const int64_t r = blockIdx.x;
    const Row row(r, p.D, 0, (int32_t)p.D);
    u32x4 x[NV], res[NV];
    row.load((const E *)p.x + r * p.D, 0, x);
    if (RES) row.load((const E *)p.r + r * p.D, 0, res);
    float yg[NV][N], sum = 0.0f;
    Largest largest;
    E *const yrow = RES ? (E *)p.y + r * p.D : nullptr;
    typename Row::Out yo{};
    if (RES) yo = row.out(yrow);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j >= row.used) continue;
        const int32_t c = row.column(j);
        float g[N];
        if (c >= 0 && c + N <= row.hi) {
            gains<N>(p, c, g);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] = c + k >= 0 && c + k < row.hi ? load_as_f32(p.g, p.g_dtype, c + k) : 0.0f;
        }
        if (RES) {
            float v[N];
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = unpack<E>(x[j], k) + unpack<E>(res[j], k);
            x[j] = pack<E>(v);                             // what is normalised is the stream as it is stored
            row.put(yo, j, x[j]);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float y = unpack<E>(x[j], k);
            sum = __builtin_fmaf(y, y, sum);
            yg[j][k] = y * g[k];
            largest.take(yg[j][k]);
        }
    }
    if (RES) row.finish(yo, yrow);
    float most = largest.value(sum);
    reduce_sum_max<T>(sum, most);
    const Scale scale(p, sum, most);
    if (threadIdx.x == 0) p.s[r] = scale.s;
    int8_t *const qrow = p.q + r * p.D;
    typename Row::OutBytes qo = row.out_bytes(qrow);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j >= row.used) continue;
        u32x2 v = {0u, 0u};
#pragma unroll
        for (int k = 0; k < N; ++k) v[k >> 2] |= (uint32_t)(scale.quantised(yg[j][k]) & 255) << (8 * (k & 3));
        row.put(qo, j, v);
    }
    row.finish(qo, qrow);
}

// rows of any length
constexpr int WG = 256;
__global__ __launch_bounds__(WG) void norm_q8_kernel(const NormQ8Params p)
{
    const int64_t row = blockIdx.x, at = row * p.D;
    float sum = 0.0f;
    Largest largest;
    for (int64_t d = threadIdx.x; d < p.D; d += WG) {
        float y = load_as_f32(p.x, p.dtype, at + d);
        if (p.r) {
            y += load_as_f32(p.r, p.dtype, at + d);
            store_from_f32(p.y, p.dtype, at + d, y);
            if (p.dtype == DT_BF16) y = round_bf16(y);
        }
        sum += y * y;
        largest.take(y * load_as_f32(p.g, p.g_dtype, d));
    }
    float most = largest.value(sum);
    reduce_sum_max<WG>(sum, most);
    const Scale scale(p, sum, most);
    if (threadIdx.x == 0) p.s[row] = scale.s;
    for (int64_t d = threadIdx.x; d < p.D; d += WG) {
        float y = load_as_f32(p.x, p.dtype, at + d);
        if (p.r) {
            y += load_as_f32(p.r, p.dtype, at + d);
            if (p.dtype == DT_BF16) y = round_bf16(y);
        }
        p.q[at + d] = (int8_t)scale.quantised(y * load_as_f32(p.g, p.g_dtype, d));
    }
}

namespace {

template <typename E, int T, int NV> void go(const NormQ8Params &p, hipStream_t s)
{
    if (p.r) hipLaunchKernelGGL((norm_q8_row_kernel<E, T, NV, true>), dim3((unsigned)p.M), dim3(T), 0, s, p);
    else hipLaunchKernelGGL((norm_q8_row_kernel<E, T, NV, false>), dim3((unsigned)p.M), dim3(T), 0, s, p);
}

// by the vectors of a row, one more for a row that begins inside one
struct Form { int64_t vecs; int threads; };
constexpr Form FORMS[] = {{64, 64}, {128, 64}, {256, 64}, {512, 256}, {1024, 256}, {4096, 1024}, {8192, 1024}, {INT64_MAX, WG}};
int form_of(const NormQ8Params &p)
{
    const int64_t n = p.dtype == DT_BF16 ? 8 : 4, vecs = (p.D + n - 1) / n + (p.D % n != 0);
    int f = 0;
    while (vecs > FORMS[f].vecs) ++f;
    return f;
}

template <typename E> void go(const NormQ8Params &p, int form, hipStream_t s)
{
    switch (form) {
    case 0: go<E, 64, 1>(p, s); break;
    case 1: go<E, 64, 2>(p, s); break;
    case 2: go<E, 64, 4>(p, s); break;
    case 3: go<E, 256, 2>(p, s); break;
    case 4: go<E, 256, 4>(p, s); break;
    case 5: go<E, 1024, 4>(p, s); break;
    case 6: go<E, 1024, 8>(p, s); break;
    default: hipLaunchKernelGGL(norm_q8_kernel, dim3((unsigned)p.M), dim3(WG), 0, s, p); break;
    }
}

}  // namespace

bool norm_q8_fits(const NormQ8Params &p) { return p.D >= 1 && launch_has(p.M, FORMS[form_of(p)].threads); }

hipError_t launch_norm_q8(const NormQ8Params &p, hipStream_t s)
{
    if (p.M < 1 || p.D < 1 || p.M > 0x7fffffff || (p.r != nullptr) != (p.y != nullptr)) return hipErrorInvalidValue;
    p.dtype == DT_BF16 ? go<uint16_t>(p, form_of(p), s) : go<float>(p, form_of(p), s);
    return hipGetLastError();
}

}  // namespace rl

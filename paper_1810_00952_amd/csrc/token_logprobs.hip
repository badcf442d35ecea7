// Log probabilities of given tokens, with entropy and the largest logits of a row, and the gradient:
//
//   m = max x,  S = sum e^(x - m),  U = sum (x - m) e^(x - m)
//   lp = x[tok] - m - ln S,   ent = ln S - U / S,   dx = dlp (1[v = tok] - p) - dent p (ln p + ent)
//
// A row of -inf alone: lp -inf, ent 0, dx 0.  A row with +inf or NaN: S is NaN, and so is everything.
//
// A workgroup holds its row in registers, as the 16-byte vectors of memory whatever the row's alignment, so that each logit is read once for
// the statistics, the alternatives and the gradient; a gradient planned right behind its forward operator shares its launch.  Every lane
// sums relative to its own maximum, the lanes' (m, S, U) meet once.  Rows too long for that, and few long rows, are cut
// into segments, whose statistics and alternatives a second launch joins.  What bounds it is HBM, and beside it two exponentials and some 19
// other vector operations a logit: 8192 x 50001 bf16 with the gradient 321 us (5.1 TB/s), 2000 x 10007 f32 28 us; four rows of 131072 bf16 with
// eight alternatives 7 and 5 us.
//
// Alternatives: each of 64 groups of lanes has its largest logit; the top-th of those is at most the top-th of the row, so what is not below it
// is collected (some 1.4 times as many as wanted) and ranked by counting.  A row where too many are not below it (equals), or that
// holds NaN, finds them one by one instead.
#include "row_vectors.h"

namespace rl {

namespace {

constexpr int CAND = 512;                        // candidates a workgroup collects
constexpr int MAX_SEGS = 64;                     // of a row
constexpr float LOWEST = -3.40282347e38f;        // the lowest number, a lane's maximum at least: -inf less it is -inf, not NaN

// maximum (at least LOWEST), S and U of x less it
struct Soft { float m, s, u; };

__device__ __forceinline__ float e_to(float x) { return __expf(x); }

__device__ __forceinline__ void rescale(Soft &a, float m)
{
    const float d = fmaxf(a.m - m, -1e4f), e = e_to(d);      // two maxima may be further apart than f32 reaches; of +inf S is NaN
    a.u = (a.u + a.s * d) * e;
    a.s *= e;
    a.m = m;
}

// of the wave's lanes, in every one of them
__device__ __forceinline__ Soft join_lanes(Soft a)
{
    rescale(a, wave_max(a.m));
    a.s = wave_sum(a.s);
    a.u = wave_sum(a.u);
    return a;
}

// the order of the alternatives as one number: larger for the larger logit, then for the earlier one; NaN above everything
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t v)
{
    uint32_t u = __float_as_uint(x + 0.0f);
    u = x != x ? 0xfffffffeu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return ((uint64_t)u << 32) | (0xffffffffu - v);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
__device__ __forceinline__ float key_logit(uint64_t key)
{
    const uint32_t u = (uint32_t)(key >> 32);
    return u == 0xfffffffeu ? __builtin_nanf("") : __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}

__device__ __forceinline__ uint64_t larger(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t largest_of_wave(uint64_t v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        v = larger(v, ((uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), o) << 32) | (uint32_t)__shfl_xor((int)(uint32_t)v, o));
    return v;
}

// a workgroup's part of a row, what is no column of it -inf
template <typename E, int T, int NV>
struct Part : RowVectors<E, T, NV> {
    typedef RowVectors<E, T, NV> Row;
    using Row::N; using Row::used;
    const E *row;                               // its column 0
    u32x4 x[NV];

    __device__ __forceinline__ Part(const void *base, int64_t r, int64_t V, int32_t lo, int32_t hi) : Row(r, V, lo, hi), row((const E *)base + r * V) {}
    __device__ __forceinline__ void load() { Row::load(row, sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u, x); }
    // the lane's own
    __device__ __forceinline__ Soft stats(float &most) const
    {
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j >= used) continue;
#pragma unroll
            for (int k = 0; k < N; ++k) m = fmaxf(m, unpack<E>(x[j], k));
        }
        most = m;
        Soft a{fmaxf(m, LOWEST), 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j >= used) continue;
            const u32x4 q = anew(x[j]);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float d = unpack<E>(q, k) - a.m, e = e_to(d);
                a.s += e;
                a.u = __builtin_fmaf(fmaxf(d, -1e4f), e, a.u);        // -inf adds zero; NaN comes with e
            }
        }
        return a;
    }
};

// statistics of all of the workgroup's lanes, in every thread; sh: one a wave
template <int T>
__device__ __forceinline__ Soft join_workgroup(Soft a, Soft *sh)
{
    a = join_lanes(a);
    if constexpr (T > 64) {
        const int lane = threadIdx.x & 63;
        if (lane == 0) sh[threadIdx.x >> 6] = a;
        __syncthreads();
        a = join_lanes(lane < T / 64 ? sh[lane] : Soft{LOWEST, 0.0f, 0.0f});
    }
    return a;
}

// what a row's results are made of
struct Result {
    float m, ls, ent, inv;
    bool dead;
    __device__ __forceinline__ explicit Result(const Soft &a)
    {
        dead = a.m == LOWEST && a.s == 0.0f;
        m = a.m;
        ls = logf(a.s);
        inv = dead ? 0.0f : 1.0f / a.s;
        ent = dead ? 0.0f : ls - a.u * inv;
    }
    __device__ __forceinline__ float logp(float x) const { return dead ? -INFINITY : x - m - ls; }
};

// the row's token, its logit and the loss' derivatives, asked for ahead of the statistics
struct Target {
    int tok;
    bool given;
    float x, dlp, dent;
    __device__ __forceinline__ Target(const LogprobsParams &p, int64_t row, bool forward, bool grad) : tok(p.tok[row])
    {
        given = tok >= 0 && tok < p.V;
        if (forward) x = load_as_f32(p.x, p.dtype, row * p.V + (given ? tok : 0));
        if (grad) { dlp = p.dlp[row]; dent = p.dent[row]; }
    }
    __device__ __forceinline__ void store(const LogprobsParams &p, int64_t row, const Result &r) const
    {
        p.lp[row] = r.ls != r.ls ? r.ls : given ? r.logp(x) : 0.0f;
        p.ent[row] = r.ent;
    }
};

// `top` keys of the workgroup's part into out (LDS), largest first; zero where there are no more.  T >= 64.
template <typename E, int T, int NV>
__device__ __forceinline__ void alternatives(const Part<E, T, NV> &x, int top, float most, bool plain, uint64_t *out)
{
    constexpr int N = Part<E, T, NV>::N, W = T / 64;
    __shared__ float group[W][64];
    __shared__ uint64_t cand[CAND], best[W];
    __shared__ int count;
    __shared__ float border;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    group[wave][lane] = most;
    if (t == 0) count = 0;
    if (t < top) out[t] = 0;
    __syncthreads();
    // the top-th largest of 64: the least of those with fewer than `top` above them
    if (wave == 0) {
        float mine = group[0][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) mine = fmaxf(mine, group[w][lane]);
        int above = 0;
#pragma unroll
        for (int l = 0; l < 64; ++l) above += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), l)) > mine;
        mine = -wave_max(above < top ? -mine : -INFINITY);
        if (lane == 0) border = mine;
    }
    __syncthreads();
    bool one_by_one = !plain;
    if (!one_by_one) {
        const float least = border;
        // fewer than `top` groups above -inf: what is above it, and for the rest the first columns, of which that many at least are -inf
        // unless what is above it is enough
        const bool some = least > -INFINITY;
        static_assert(CAND / 2 >= 2 * LOGPROBS_MAX_TOP, "columns that hold `top` logits beside fewer than `top`");
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (j >= x.used) continue;
            const u32x4 q = anew(x.x[j]);
            float f[N], v = -INFINITY;
#pragma unroll
            for (int k = 0; k < N; ++k) { f[k] = unpack<E>(q, k); v = fmaxf(v, f[k]); }
            if (v >= least) {
                const int32_t c = anew(x.column(j));
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (f[k] >= least && (some || f[k] > -INFINITY || c + k < x.lo + CAND / 2) && c + k >= x.lo && c + k < x.hi) {
                        const int at = atomicAdd(&count, 1);
                        if (at < CAND) cand[at] = rank_key(f[k], (uint32_t)(c + k));
                    }
            }
        }
        __syncthreads();
        const int n = count;
        one_by_one = n > CAND;
        if (!one_by_one)
            for (int i = t; i < n; i += T) {
                const uint64_t key = cand[i];
                int rank = 0;
                for (int o = 0; o < n; ++o) rank += cand[o] > key;
                if (rank < top) out[rank] = key;
            }
    }
    if (one_by_one) {
        uint64_t last = ~(uint64_t)0;
        for (int i = 0; i < top; ++i) {
            uint64_t b = 0;                          // below every key: a column is under 2^31
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (j >= x.used) continue;
                const int32_t c = anew(x.column(j));
                const u32x4 q = anew(x.x[j]);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const uint64_t key = rank_key(unpack<E>(q, k), (uint32_t)(c + k));
                    if (key < last && c + k >= x.lo && c + k < x.hi) b = larger(b, key);
                }
            }
            b = largest_of_wave(b);
            if (lane == 0) best[wave] = b;
            __syncthreads();
            for (int w = 0; w < W; ++w) b = larger(b, best[w]);
            last = b;
            if (t == 0) out[i] = b;
            __syncthreads();
            if (b == 0) break;
        }
    }
    __syncthreads();
}

template <typename E, int T, int NV>
__device__ __forceinline__ void gradient(const LogprobsParams &p, const Part<E, T, NV> &x, int64_t row, const Result &r, const Target &target)
{
    constexpr int N = Part<E, T, NV>::N;
    const int tok = target.tok;
    const float dlp = target.given && !r.dead ? target.dlp : 0.0f;
    const float dent = r.dead ? 0.0f : -r.inv * target.dent, c = r.dead ? 0.0f : __builtin_fmaf(dent, r.ent - r.ls, -r.inv * dlp);
    // whose the token is
    const int32_t tok_v = (tok - x.first) / N, tok_k = (tok - x.first) % N, tok_j = tok < x.lo || tok >= x.hi ? -1 : tok_v / T;
    const uint32_t tok_t = (uint32_t)(tok_v % T);
    E *dx = (E *)p.dx + row * p.V;
    auto out = x.out(dx);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j >= x.used) continue;
        const u32x4 q = anew(x.x[j]);
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float d = unpack<E>(q, k) - r.m;
            v[k] = e_to(d) * __builtin_fmaf(dent, fmaxf(d, -1e4f), c);
        }
        if (j == tok_j && threadIdx.x == tok_t) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k == tok_k) v[k] += dlp;
        }
        x.put(out, j, pack<E>(v));
    }
    x.finish(out, dx);
}

// What a segment leaves in part for the second launch: m, S, U, -, then `top` keys
__device__ __forceinline__ int64_t seg_floats(int top) { return 4 + 2 * top; }

__device__ __forceinline__ Soft join_segments(const LogprobsParams &p, int64_t row, int segs)
{
    static_assert(MAX_SEGS <= 64, "a lane each");
    const int lane = threadIdx.x & 63;
    const float *v = p.part + (row * segs + lane) * seg_floats(p.top);
    return join_lanes(lane < segs ? Soft{v[0], v[1], v[2]} : Soft{LOWEST, 0.0f, 0.0f});
}

enum { FORWARD = 1, GRADIENT = 2, SEGMENT = 4, JOINED = 8, TOP = 16 };     // what a launch does: JOINED takes the statistics from part, TOP: p.top > 0

}  // namespace

template <typename E, int T, int NV, int WHAT>
__global__ __launch_bounds__(T, NV == 16 ? 4 : 8) void token_logprobs_kernel(const LogprobsParams p, int32_t segs, int32_t seg_len)
{
    __shared__ Soft sh[T / 64];
    __shared__ uint64_t keys[LOGPROBS_MAX_TOP];
    const int64_t row = blockIdx.x / (uint32_t)segs;
    const int32_t seg = (int32_t)(blockIdx.x - (uint32_t)row * segs), lo = seg * seg_len;
    Part<E, T, NV> x(p.x, row, p.V, lo, (int32_t)min((int64_t)lo + seg_len, p.V));
    x.load();
    const Target target(p, row, WHAT & FORWARD, WHAT & GRADIENT);
    float most = 0.0f;
    const Soft a = WHAT & JOINED ? join_segments(p, row, segs) : join_workgroup<T>(x.stats(most), sh);
    if constexpr (WHAT & TOP) alternatives<E, T, NV>(x, p.top, most, a.s == a.s, keys);
    if constexpr (WHAT & SEGMENT) {
        float *q = p.part + (row * segs + seg) * seg_floats(p.top);
        if (threadIdx.x == 0) { q[0] = a.m; q[1] = a.s; q[2] = a.u; }
        if (WHAT & TOP && (int)threadIdx.x < p.top) ((uint64_t *)(q + 4))[threadIdx.x] = keys[threadIdx.x];
        return;
    }
    const Result r(a);
    if constexpr (WHAT & FORWARD) {
        if (threadIdx.x == 0) target.store(p, row, r);
        if (WHAT & TOP && (int)threadIdx.x < p.top) {
            const uint64_t key = keys[threadIdx.x];
            p.top_id[row * p.top + threadIdx.x] = (int32_t)key_index(key);
            p.top_lp[row * p.top + threadIdx.x] = r.logp(key_logit(key));
        }
    }
    if constexpr (WHAT & GRADIENT) gradient<E, T, NV>(p, x, row, r, target);
}

// the segments of a row joined, their alternatives ranked by counting those that can be among the row's
__global__ __launch_bounds__(256) void token_logprobs_join_kernel(const LogprobsParams p, int32_t segs)
{
    __shared__ uint64_t keys[MAX_SEGS * LOGPROBS_MAX_TOP], cand[MAX_SEGS * LOGPROBS_MAX_TOP], least;
    __shared__ int count;
    const int64_t row = blockIdx.x;
    const float *q = p.part + row * segs * seg_floats(p.top);
    const int n = segs * p.top, t = threadIdx.x;
    for (int i = t; i < n; i += 256) keys[i] = ((const uint64_t *)(q + (i / p.top) * seg_floats(p.top) + 4))[i % p.top];
    if (t == 0) count = 0;
    const Target target(p, row, true, false);
    const Result r(join_segments(p, row, segs));
    if (t == 0) target.store(p, row, r);
    if (p.top == 0) return;
    __syncthreads();
    // the top-th of the segments' first `each`, which are `top` or a few more: nothing below it is wanted
    const int each = (p.top + segs - 1) / segs, some = segs * each;
    static_assert(MAX_SEGS + LOGPROBS_MAX_TOP <= 256, "a thread each");
    if (t < some) {
        const uint64_t key = keys[t / each * p.top + t % each];
        int rank = 0;
        for (int s = 0; s < segs; ++s)
            for (int k = 0; k < each; ++k) {
                const uint64_t other = keys[s * p.top + k];
                rank += other > key || (other == key && s * each + k < t);          // equal: the zeros of a segment with fewer
            }
        if (rank == p.top - 1) least = key;
    }
    __syncthreads();
    for (int i = t; i < n; i += 256)
        if (keys[i] >= least && keys[i] != 0) cand[atomicAdd(&count, 1)] = keys[i];
    __syncthreads();
    for (int i = t; i < count; i += 256) {
        const uint64_t key = cand[i];
        int rank = 0;
        for (int o = 0; o < count; ++o) rank += cand[o] > key;
        if (rank < p.top) {
            p.top_id[row * p.top + rank] = (int32_t)key_index(key);
            p.top_lp[row * p.top + rank] = r.logp(key_logit(key));
        }
    }
}

// ---------------------------------------------------------------------------
namespace {

struct Form { int segs; int32_t len; int shape; };           // shape: of the kernel, by the bytes it holds

constexpr int SHAPE_THREADS[] = {64, 256, 512, 1024, 1024};
constexpr int64_t SHAPE_BYTES[] = {64 * 4 * 16, 256 * 4 * 16, 512 * 8 * 16, 1024 * 8 * 16, 1024 * 16 * 16};

Form form_of(const LogprobsParams &p)
{
    const int64_t e = p.dtype == DT_BF16 ? 2 : 4;
    Form f{1, (int32_t)p.V, 0};
    // a row that is not cut, or segments of 16 KB: enough for all CUs where there are few rows
    const int64_t most = SHAPE_BYTES[4] - 16;                  // 16: a row may begin inside a vector
    if (p.V * e > most || (p.M < 128 && p.V * e > 32768)) {
        int64_t segs = p.M < 128 ? (256 + p.M - 1) / p.M : 1;
        segs = segs < p.V * e / 16000 + 1 ? segs : p.V * e / 16000 + 1;
        if (segs > MAX_SEGS) segs = MAX_SEGS;
        const int64_t need = (p.V * e + most - 1) / most;
        if (segs < need) segs = need;
        f.len = (int32_t)((p.V + segs - 1) / segs);
        f.segs = (int)((p.V + f.len - 1) / f.len);
    }
    while (f.shape < 4 && f.len * e + 16 > SHAPE_BYTES[f.shape]) ++f.shape;
    return f;
}

template <typename E, int T, int NV>
void go(const LogprobsParams &p, const Form &f, int what, hipStream_t s)
{
    const dim3 grid((unsigned)(p.M * f.segs)), wg(T);
#define RL_GO(WHAT) case WHAT: hipLaunchKernelGGL((token_logprobs_kernel<E, T, NV, WHAT>), grid, wg, 0, s, p, f.segs, f.len); break;
    switch (what) {
        RL_GO(FORWARD) RL_GO(FORWARD | TOP) RL_GO(GRADIENT) RL_GO(FORWARD | GRADIENT) RL_GO(FORWARD | GRADIENT | TOP)
        RL_GO(SEGMENT) RL_GO(SEGMENT | TOP) RL_GO(GRADIENT | JOINED)
    }
#undef RL_GO
}

template <typename E>
void go(const LogprobsParams &p, const Form &f, int what, hipStream_t s)
{
    switch (f.shape) {
    case 0: go<E, 64, 4>(p, f, what, s); break;
    case 1: go<E, 256, 4>(p, f, what, s); break;
    case 2: go<E, 512, 8>(p, f, what, s); break;
    case 3: go<E, 1024, 8>(p, f, what, s); break;
    default: go<E, 1024, 16>(p, f, what, s); break;
    }
}

}  // namespace

int64_t logprobs_part_floats(const LogprobsParams &p)
{
    const Form f = form_of(p);
    return f.segs > 1 ? p.M * f.segs * (4 + 2 * (int64_t)p.top) : 0;
}

bool logprobs_fits(const LogprobsParams &p)
{
    if (p.M < 1 || p.V < 1 || p.M > 0x7fffffff || p.V > LOGPROBS_MAX_V) return false;
    const Form f = form_of(p);
    return f.segs <= MAX_SEGS && f.len * (p.dtype == DT_BF16 ? 2 : 4) + 16 <= SHAPE_BYTES[4] && launch_has(p.M * f.segs, SHAPE_THREADS[f.shape]);      // the joining launch has no more
}

hipError_t launch_logprobs(const LogprobsParams &p, bool forward, bool grad, hipStream_t s)
{
    const Form f = form_of(p);
    if (p.M < 1 || p.V < 1 || p.V > LOGPROBS_MAX_V || f.segs > MAX_SEGS || p.M * f.segs > 0x7fffffff || f.len * (p.dtype == DT_BF16 ? 2 : 4) + 16 > SHAPE_BYTES[4] ||
        p.top < 0 || p.top > p.V || p.top > LOGPROBS_MAX_TOP || (f.segs > 1 && !p.part)) return hipErrorInvalidValue;
    auto run = [&](int what) { p.dtype == DT_BF16 ? go<uint16_t>(p, f, what, s) : go<float>(p, f, what, s); };
    if (f.segs == 1) {
        run((forward ? FORWARD : 0) | (grad ? GRADIENT : 0) | (forward && p.top > 0 ? TOP : 0));
    } else {
        run(SEGMENT | (forward && p.top > 0 ? TOP : 0));
        if (forward) hipLaunchKernelGGL(token_logprobs_join_kernel, dim3((unsigned)p.M), dim3(256), 0, s, p, f.segs);
        if (grad) run(GRADIENT | JOINED);
    }
    return hipGetLastError();
}

}  // namespace rl

// Selective state-space scan: every channel d has N numbers of state, and every token its own gates,
//
//   s = softplus(dt[t,d]),   h_t[d,n] = exp(s a[d,n]) h_(t-1)[d,n] + s x[t,d] B[t,n],   y[t,d] = (sum_n C[t,n] h_t[d,n] + skip[d] x[t,d]) z sigmoid(z)
//
// and its gradient, with du = dy z sigmoid(z): G_t[d,n] = C[t,n] du[t,d] + exp(s_(t+1) a) G_(t+1),
//   dB[t,n] = sum_d G s x,  dC[t,n] = sum_d du h,  dx = skip du + s sum_n G B,  da = sum_t G h_(t-1) exp(s a) s,
//   ds = sum_n G (h_(t-1) exp(s a) a + x B),  ddt = ds sigmoid(dt).
//
// Four states of a channel are a lane's, L lanes a channel's (N <= 4 L), 256 / L channels a workgroup's, which walks the rows by tiles: what a
// channel needs once a token (softplus, the gate, products) is found by a thread a token and channel, and meets the states in LDS.  A row that is
// padding has s = s x = B = C = du = 0 and leaves state and derivative as they are.  Few channels: the rows are cut into chunks, a workgroup
// each; a launch ahead finds what each chunk makes of the state before it (P h + H; the derivative alike), P = exp(a sum s), and the workgroups
// add up the chunks before theirs.
#include "igemm_lds.h"

namespace rl {

namespace {

constexpr int R = 4;                          // states of a lane
constexpr int ROWS = SSM_STATE_ROWS;          // rows of a tile
constexpr float LOG2E = 1.4426950408889634f;

// Chunks' P of which a document's first row is part: -0, which no product of gates is
constexpr float FIRST = -0.0f;
__device__ __forceinline__ bool is_first(float P) { return __float_as_uint(P) == 0x80000000u; }
__device__ __forceinline__ float through(float P, float h, float H)
{
    const float y = __builtin_fmaf(P, h, H);
    return is_first(P) ? H : y;
}
__device__ __forceinline__ float exp2_(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(v);
#else
    return v;
#endif
}

// ln(1 + e^v): for large v it is v; below, with w = e^v, ln(1 + w) w / ((1 + w) - 1) keeps its last bits where 1 + w loses those of w
__device__ __forceinline__ float softplus(float v)
{
    const float w = __expf(v), u = 1.0f + w;
    const float small = u == 1.0f ? w : __logf(u) * (w * rcp_(u - 1.0f));
    return v > 20.0f ? v : small;
}

template <typename E> __device__ __forceinline__ float at(const void *p, int64_t i)
{
    if constexpr (sizeof(E) == 4) return ((const float *)p)[i];
    else return bf16_bits_to_f32(((const uint16_t *)p)[i]);
}
template <typename E> __device__ __forceinline__ void put(void *p, int64_t i, float v)
{
    if constexpr (sizeof(E) == 4) ((float *)p)[i] = v;
    else ((uint16_t *)p)[i] = (uint16_t)pack_bf16x2(v, v);
}

// sum over a channel's lanes, in all of them
template <int L> __device__ __forceinline__ float over_states(float v)
{
#pragma unroll
    for (int k = 1; k < L; k <<= 1) v += __shfl_xor(v, k);
    return v;
}
// sum over a wave's channels, in all lanes
template <int L> __device__ __forceinline__ float over_channels(float v)
{
#pragma unroll
    for (int k = L; k < 64; k <<= 1) v += __shfl_xor(v, k);
    return v;
}

// what a lane works on
template <int L>
struct Place {
    static constexpr int CH = 256 / L;        // channels of a workgroup
    static constexpr int EACH = ROWS / L;     // rows a thread does the token-and-channel work of (every 256 / CH-th)
    int l, c, pc, pr;                         // the states' lane: its states l R .., channel c; the channel and first row of the work a token
    int64_t b, d, pd;                         // ... their numbers in the sequence's rows
    int32_t chunk, slab;
    bool live, plive;
    __device__ __forceinline__ Place(const SelScanParams &p, int32_t slabs)
    {
        l = threadIdx.x % L; c = threadIdx.x / L;
        pc = threadIdx.x % CH; pr = threadIdx.x / CH;
        const uint32_t rest = blockIdx.x / (uint32_t)slabs;
        slab = (int32_t)(blockIdx.x - rest * slabs);
        chunk = (int32_t)(rest / (uint32_t)p.B);
        b = rest - (uint32_t)chunk * (uint32_t)p.B;
        d = (int64_t)slab * CH + c; pd = (int64_t)slab * CH + pc;
        live = d < p.D; plive = pd < p.D;
        if (!live) d = 0;                     // some other channel's, of which nothing is stored
        if (!plive) pd = 0;
    }
    // R numbers of a [D][N] matrix (rest for the states behind N)
    __device__ __forceinline__ void load(const SelScanParams &p, const float *m, float (&v)[R], float rest = 0.0f) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = l * R + r < p.N ? m[d * p.N + l * R + r] : rest;
    }
    __device__ __forceinline__ void store(const SelScanParams &p, float *m, const float (&v)[R]) const
    {
        if (!live) return;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l * R + r < p.N) m[d * p.N + l * R + r] = v[r];
    }
};

// rows of a tile that are tokens, that are a document's first
template <bool KEEP> __device__ __forceinline__ void flags_of(const SelScanParams &p, int64_t b, int64_t t0, uint32_t &tok, uint32_t &first)
{
    const int i = threadIdx.x & 63;
    const bool in = i < ROWS && t0 + i < p.T;
    const int k = !in ? 0 : KEEP ? p.keep[b * p.T + t0 + i] : 1;
    tok = (uint32_t)__ballot(k != 0);
    first = KEEP ? (uint32_t)__ballot(k == 2) : 0;
}

// B and C of a tile's rows, zeros behind N and of padding
template <typename E, int L> __device__ __forceinline__ void stage_bc(const SelScanParams &p, int64_t row0, uint32_t tok, float (&sb)[2][ROWS][4 * L])
{
    for (int i = threadIdx.x; i < ROWS * 8 * L; i += 256) {
        const int n = i % (4 * L), t = i / (4 * L) % ROWS, which = i / (4 * L * ROWS);
        sb[which][t][n] = (tok >> t & 1) && n < p.N ? at<E>(p.bc, (row0 + t) * 2 * p.N + which * p.N + n) : 0.0f;
    }
}

}  // namespace

// ---------------------------------------------------------------------------
// one token a sequence
// ---------------------------------------------------------------------------
template <typename E, int L>
__global__ __launch_bounds__(256) void selective_scan_step_kernel(const SelScanParams p, int64_t channels)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int l = threadIdx.x % L;
    const bool live = i < channels;
    const int64_t c = live ? i : 0, b = c / p.D, d = c - b * p.D;
    const int keep = p.keep ? p.keep[b] : 1;
    const float x = keep ? at<E>(p.x, c) : 0.0f, s = keep ? softplus(at<E>(p.dt, c)) : 0.0f, v = s * x;
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int n = l * R + r;
        if (n >= p.N) continue;
        const float h0 = p.h0[c * p.N + n], e = exp2_(s * (p.a[d * p.N + n] * LOG2E));
        const float u = keep ? v * at<E>(p.bc, b * 2 * p.N + n) : 0.0f;
        const float h = keep == 2 ? u : keep ? __builtin_fmaf(e, h0, u) : h0;
        if (live) p.hT[c * p.N + n] = h;
        sum = __builtin_fmaf(keep ? at<E>(p.bc, (b * 2 + 1) * p.N + n) : 0.0f, h, sum);
    }
    sum = over_states<L>(sum);
    if (l == 0 && live) {
        float y = __builtin_fmaf(p.skip[d], x, sum);
        if (p.z) { const float z = at<E>(p.z, c); y *= z * sigmoidf_(z); }
        put<E>(p.y, c, keep ? y : 0.0f);
    }
}

// ---------------------------------------------------------------------------
// forward.  AHEAD: what a chunk makes of the state before it, into part ([chunk][b] P, H of [D][N])
// ---------------------------------------------------------------------------
template <typename E, int L, bool KEEP, bool AHEAD>
__global__ __launch_bounds__(256) void selective_scan_kernel(const SelScanParams p, int32_t slabs, int32_t chunks, int32_t chunk_tiles)
{
    typedef Place<L> P;
    constexpr int CH = P::CH, EACH = P::EACH;
    const P at_(p, slabs);
    const int64_t DN = p.D * p.N;
    __shared__ float2 sd[ROWS][CH];                                  // s, s x
    __shared__ __attribute__((aligned(16))) float sb[2][ROWS][4 * L];
    __shared__ float sy[ROWS][CH];
    float a2[R], h[R], total = 0.0f;
    at_.load(p, p.a, a2);
#pragma unroll
    for (int r = 0; r < R; ++r) { a2[r] *= LOG2E; h[r] = 0.0f; }
    bool began = false;                                              // a document's first row was there
    if (!AHEAD) {
        at_.load(p, p.h0 + at_.b * DN, h);
        for (int32_t k = 0; k < at_.chunk; ++k) {
            float f[R], H[R];
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b)) * DN, f);
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b) + 1) * DN, H);
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = through(f[r], h[r], H[r]);
        }
    }
    const float skip = p.skip[at_.pd];
    const int64_t tiles = (p.T + ROWS - 1) / ROWS;
    const int64_t first_tile = (int64_t)at_.chunk * chunk_tiles, end_tile = min(first_tile + chunk_tiles, tiles);
    for (int64_t tile = first_tile; tile < end_tile; ++tile) {
        const int64_t t0 = tile * ROWS, row0 = at_.b * p.T + t0;
        uint32_t tok, first;
        flags_of<KEEP>(p, at_.b, t0, tok, first);
        float x[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int t = at_.pr + e * L;
            const bool here = tok >> t & 1;
            x[e] = here ? at<E>(p.x, (row0 + t) * p.D + at_.pd) : 0.0f;
            const float s = here ? softplus(at<E>(p.dt, (row0 + t) * p.D + at_.pd)) : 0.0f;
            sd[t][at_.pc] = float2{s, s * x[e]};
        }
        stage_bc<E, L>(p, row0, tok, sb);
        __syncthreads();
        if (p.states && !AHEAD) at_.store(p, p.states + (at_.b * tiles + tile) * DN, h);
#pragma unroll
        for (int t = 0; t < ROWS; ++t) {
            const float2 sv = sd[t][at_.c];
            if (KEEP && (first >> t & 1)) {
                began = true;
#pragma unroll
                for (int r = 0; r < R; ++r) h[r] = 0.0f;
            }
            if (AHEAD) total += sv.x;
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                h[r] = __builtin_fmaf(exp2_(sv.x * a2[r]), h[r], sv.y * sb[0][t][at_.l * R + r]);
                if (!AHEAD) sum = __builtin_fmaf(sb[1][t][at_.l * R + r], h[r], sum);
            }
            if (!AHEAD) {
                sum = over_states<L>(sum);
                if (at_.l == 0) sy[t][at_.c] = sum;
            }
        }
        __syncthreads();
        if (!AHEAD && p.y) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int t = at_.pr + e * L;
                if (t0 + t >= p.T || !at_.plive) continue;
                const int64_t i = (row0 + t) * p.D + at_.pd;
                float y = __builtin_fmaf(skip, x[e], sy[t][at_.pc]);
                if (p.z) { const float z = at<E>(p.z, i); y *= z * sigmoidf_(z); }
                put<E>(p.y, i, tok >> t & 1 ? y : 0.0f);
            }
        }
    }
    if (AHEAD) {
        float f[R];
#pragma unroll
        for (int r = 0; r < R; ++r) f[r] = began ? FIRST : exp2_(fmaxf(total * a2[r], -126.0f));
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b)) * DN, f);
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b) + 1) * DN, h);
    } else if (p.hT && at_.chunk + 1 == chunks) {
        at_.store(p, p.hT + at_.b * DN, h);
    }
}

// ---------------------------------------------------------------------------
// gradient, tiles from the last to the first.  AHEAD: what a chunk makes of the derivative behind it, into part
// ---------------------------------------------------------------------------
template <typename E, int L, bool KEEP, bool AHEAD>
__global__ __launch_bounds__(256) void selective_scan_grad_kernel(const SelScanParams p, int32_t slabs, int32_t chunks, int32_t chunk_tiles, float *shares, float *bc_shares)
{
    typedef Place<L> P;
    constexpr int CH = P::CH, EACH = P::EACH;
    const P at_(p, slabs);
    const int64_t DN = p.D * p.N;
    __shared__ __attribute__((aligned(16))) float4 sd[ROWS][CH];     // s, s x, du
    __shared__ __attribute__((aligned(16))) float sb[2][ROWS][4 * L];
    __shared__ float ss[3][ROWS][CH];                                // sum of G B, of G h exp(s a) a, of C h
    __shared__ float sc[4][2][ROWS][4 * L];                          // dB, dC of a wave's channels
    const int wave = threadIdx.x >> 6;
    float a[R], G[R], da[R], total = 0.0f, dskip = 0.0f;
    at_.load(p, p.a, a);
#pragma unroll
    for (int r = 0; r < R; ++r) { G[r] = 0.0f; da[r] = 0.0f; }
    bool began = false;
    if (!AHEAD) {
        at_.load(p, p.dhT + at_.b * DN, G);
        for (int32_t k = chunks - 1; k > at_.chunk; --k) {
            float f[R], H[R];
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b)) * DN, f);
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b) + 1) * DN, H);
#pragma unroll
            for (int r = 0; r < R; ++r) G[r] = through(f[r], G[r], H[r]);
        }
    }
    const float skip = p.skip[at_.pd];
    const int64_t tiles = (p.T + ROWS - 1) / ROWS;
    const int64_t first_tile = (int64_t)at_.chunk * chunk_tiles, end_tile = min(first_tile + chunk_tiles, tiles);
    for (int64_t tile = end_tile - 1; tile >= first_tile; --tile) {
        const int64_t t0 = tile * ROWS, row0 = at_.b * p.T + t0;
        uint32_t tok, first;
        flags_of<KEEP>(p, at_.b, t0, tok, first);
        float x[EACH], dt[EACH], dy[EACH], z[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int t = at_.pr + e * L;
            const bool here = tok >> t & 1;
            const int64_t i = (row0 + t) * p.D + at_.pd;
            x[e] = here ? at<E>(p.x, i) : 0.0f;
            dt[e] = here ? at<E>(p.dt, i) : 0.0f;
            dy[e] = here ? at<E>(p.dy, i) : 0.0f;
            z[e] = here && p.z ? at<E>(p.z, i) : 0.0f;
            const float s = here ? softplus(dt[e]) : 0.0f, du = p.z ? dy[e] * (z[e] * sigmoidf_(z[e])) : dy[e];
            sd[t][at_.pc] = float4{s, s * x[e], du, 0.0f};
            if (!AHEAD) dskip = __builtin_fmaf(du, x[e], dskip);
        }
        stage_bc<E, L>(p, row0, tok, sb);
        __syncthreads();
        if (AHEAD) {
#pragma unroll
            for (int t = ROWS - 1; t >= 0; --t) {
                const float4 v = sd[t][at_.c];
                total += v.x;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    G[r] = __builtin_fmaf(sb[1][t][at_.l * R + r], v.z, G[r]) * exp2_(v.x * (a[r] * LOG2E));
                    if (KEEP && (first >> t & 1)) G[r] = 0.0f;
                }
            }
            began |= KEEP && first != 0;
        } else {
            float h[R], before[ROWS][R], gate[ROWS][R];
            at_.load(p, p.states + (at_.b * tiles + tile) * DN, h);
#pragma unroll
            for (int t = 0; t < ROWS; ++t) {
                const float4 v = sd[t][at_.c];
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (KEEP && (first >> t & 1)) h[r] = 0.0f;
                    before[t][r] = h[r];
                    gate[t][r] = exp2_(v.x * (a[r] * LOG2E));
                    h[r] = __builtin_fmaf(gate[t][r], h[r], v.y * sb[0][t][at_.l * R + r]);
                    sum = __builtin_fmaf(sb[1][t][at_.l * R + r], h[r], sum);
                }
                if (p.z) {
                    sum = over_states<L>(sum);
                    if (at_.l == 0) ss[2][t][at_.c] = sum;
                }
            }
#pragma unroll
            for (int t = ROWS - 1; t >= 0; --t) {
                const float4 v = sd[t][at_.c];
                float gb = 0.0f, ga = 0.0f, db[R], dc[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float B = sb[0][t][at_.l * R + r], he = before[t][r] * gate[t][r];
                    G[r] = __builtin_fmaf(sb[1][t][at_.l * R + r], v.z, G[r]);
                    const float arg = G[r] * he;
                    da[r] = __builtin_fmaf(arg, v.x, da[r]);
                    ga = __builtin_fmaf(arg, a[r], ga);
                    gb = __builtin_fmaf(G[r], B, gb);
                    db[r] = at_.live ? G[r] * v.y : 0.0f;
                    dc[r] = at_.live ? v.z * __builtin_fmaf(v.y, B, he) : 0.0f;
                    G[r] *= gate[t][r];
                    if (KEEP && (first >> t & 1)) G[r] = 0.0f;
                }
                gb = over_states<L>(gb);
                ga = over_states<L>(ga);
                if (at_.l == 0) { ss[0][t][at_.c] = gb; ss[1][t][at_.c] = ga; }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    db[r] = over_channels<L>(db[r]);
                    dc[r] = over_channels<L>(dc[r]);
                    if ((threadIdx.x & 63) < L) { sc[wave][0][t][at_.l * R + r] = db[r]; sc[wave][1][t][at_.l * R + r] = dc[r]; }
                }
            }
        }
        __syncthreads();
        if (!AHEAD) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int t = at_.pr + e * L;
                if (t0 + t >= p.T || !at_.plive) continue;
                const bool here = tok >> t & 1;
                const int64_t i = (row0 + t) * p.D + at_.pd;
                const float4 v = sd[t][at_.pc];
                const float gb = ss[0][t][at_.pc], ga = ss[1][t][at_.pc];
                put<E>(p.dx, i, here ? __builtin_fmaf(skip, v.z, v.x * gb) : 0.0f);
                put<E>(p.ddt, i, here ? __builtin_fmaf(x[e], gb, ga) * sigmoidf_(dt[e]) : 0.0f);
                if (p.z) {
                    const float s = sigmoidf_(z[e]), u = __builtin_fmaf(skip, x[e], ss[2][t][at_.pc]);
                    put<E>(p.dz, i, here ? dy[e] * u * __builtin_fmaf(z[e] * s, sigmoidf_(-z[e]), s) : 0.0f);
                }
            }
            for (int i = threadIdx.x; i < ROWS * 2 * (int)p.N; i += 256) {
                const int n = i % (int)p.N, which = i / (int)p.N % 2, t = i / (2 * (int)p.N);
                if (t0 + t >= p.T) continue;
                float sum = sc[0][which][t][n];
#pragma unroll
                for (int w = 1; w < 4; ++w) sum += sc[w][which][t][n];
                bc_shares[((int64_t)at_.slab * p.B * p.T + row0 + t) * 2 * p.N + which * p.N + n] = tok >> t & 1 ? sum : 0.0f;
            }
        }
    }
    if (AHEAD) {
        float f[R];
#pragma unroll
        for (int r = 0; r < R; ++r) f[r] = began ? FIRST : exp2_(fmaxf(total * (a[r] * LOG2E), -126.0f));
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b)) * DN, f);
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b) + 1) * DN, G);
        return;
    }
    if (at_.chunk == 0) at_.store(p, p.dh0 + at_.b * DN, G);
    float *mine = shares + ((int64_t)at_.chunk * p.B + at_.b) * (DN + p.D);
    at_.store(p, mine, da);
    // the threads of a channel's tokens add up what they have of dskip
    __syncthreads();
    float *const sums = &ss[0][0][0];
    sums[at_.pr * CH + at_.pc] = dskip;
    __syncthreads();
    if (at_.pr == 0 && at_.plive) {
        for (int k = 1; k < L; ++k) dskip += sums[k * CH + at_.pc];
        mine[DN + at_.pd] = dskip;
    }
}

namespace {

struct Form { int L; int32_t slabs, chunks, chunk_tiles; };

Form form_of(const SelScanParams &p)
{
    Form f;
    f.L = 1;
    while (f.L * R < p.N) f.L *= 2;
    const int64_t ch = 256 / f.L, tiles = (p.T + ROWS - 1) / ROWS;
    f.slabs = (int32_t)((p.D + ch - 1) / ch);
    const int64_t wgs = p.B * f.slabs;
    int64_t chunks = 1;
    if (wgs < 256) chunks = 512 / wgs;
    if (chunks > tiles / 4) chunks = tiles / 4 > 0 ? tiles / 4 : 1;
    f.chunk_tiles = (int32_t)((tiles + chunks - 1) / chunks);
    f.chunks = (int32_t)((tiles + f.chunk_tiles - 1) / f.chunk_tiles);
    return f;
}

struct Scratch { int64_t chunks, shares, bc; };          // floats of each
Scratch scratch_of(const SelScanParams &p, const Form &f, bool grad)
{
    Scratch s{};
    s.chunks = f.chunks > 1 ? 2 * f.chunks * p.B * p.D * p.N : 0;
    if (grad) {
        s.shares = f.chunks * p.B * (p.D * p.N + p.D);
        s.bc = f.slabs * p.B * p.T * 2 * p.N;
    }
    return s;
}

template <typename E, int L>
hipError_t go(bool grad, const SelScanParams &p, const Form &f, hipStream_t s)
{
    const dim3 grid((unsigned)(p.B * f.slabs * f.chunks)), wg(256);
    if (!grad) {
        if (f.chunks > 1) {
            if (p.keep) hipLaunchKernelGGL((selective_scan_kernel<E, L, true, true>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles);
            else hipLaunchKernelGGL((selective_scan_kernel<E, L, false, true>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles);
        }
        if (p.keep) hipLaunchKernelGGL((selective_scan_kernel<E, L, true, false>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles);
        else hipLaunchKernelGGL((selective_scan_kernel<E, L, false, false>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles);
        return hipGetLastError();
    }
    const Scratch sc = scratch_of(p, f, true);
    float *const shares = p.part + sc.chunks, *const bc = shares + sc.shares;
    if (f.chunks > 1) {
        if (p.keep) hipLaunchKernelGGL((selective_scan_grad_kernel<E, L, true, true>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles, shares, bc);
        else hipLaunchKernelGGL((selective_scan_grad_kernel<E, L, false, true>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles, shares, bc);
    }
    if (p.keep) hipLaunchKernelGGL((selective_scan_grad_kernel<E, L, true, false>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles, shares, bc);
    else hipLaunchKernelGGL((selective_scan_grad_kernel<E, L, false, false>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_tiles, shares, bc);
    hipError_t er = hipGetLastError();
    if (er != hipSuccess) return er;
    SumShares q{};
    q.part = shares; q.P = f.chunks * p.B; q.stride = p.D * p.N + p.D; q.dst_dtype = DT_F32;
    q.J = p.D * p.N; q.dst = p.da;
    er = launch_sum_shares(q, s);
    if (er != hipSuccess) return er;
    q.part = shares + p.D * p.N; q.J = p.D; q.dst = p.dskip;
    er = launch_sum_shares(q, s);
    if (er != hipSuccess) return er;
    q.part = bc; q.P = f.slabs; q.J = q.stride = p.B * p.T * 2 * p.N; q.dst = p.dbc; q.dst_dtype = p.dtype;
    return launch_sum_shares(q, s);
}

template <typename E> hipError_t go(bool grad, const SelScanParams &p, const Form &f, hipStream_t s)
{
    switch (f.L) {
    case 1: return go<E, 1>(grad, p, f, s);
    case 2: return go<E, 2>(grad, p, f, s);
    case 4: return go<E, 4>(grad, p, f, s);
    case 8: return go<E, 8>(grad, p, f, s);
    default: return go<E, 16>(grad, p, f, s);
    }
}

template <typename E, int L> void go_step(const SelScanParams &p, hipStream_t s)
{
    const int64_t channels = p.B * p.D;
    hipLaunchKernelGGL((selective_scan_step_kernel<E, L>), dim3((unsigned)((channels * L + 255) / 256)), dim3(256), 0, s, p, channels);
}
template <typename E> hipError_t go_step(const SelScanParams &p, int L, hipStream_t s)
{
    switch (L) {
    case 1: go_step<E, 1>(p, s); break;
    case 2: go_step<E, 2>(p, s); break;
    case 4: go_step<E, 4>(p, s); break;
    case 8: go_step<E, 8>(p, s); break;
    default: go_step<E, 16>(p, s); break;
    }
    return hipGetLastError();
}

}  // namespace

bool sel_scan_fits(const SelScanParams &p, bool grad)
{
    if (p.B < 1 || p.T < 1 || p.D < 1 || p.N < 1 || p.N > SSM_MAX_STATES || p.B > 0x7fffffff || p.T > 0x7fffffff || p.D > SCAN_MAX_D) return false;
    const Form f = form_of(p);
    if (p.T == 1 && !grad) return launch_has((p.B * p.D * f.L + 255) / 256, 256);
    // the sums over channels are a launch of a thousand threads a 64 columns
    return launch_has(p.B * f.slabs * f.chunks, 256) && (!grad || (p.B * p.T * 2 * p.N + 63) / 64 <= 0x3fffff);
}

int64_t sel_scan_part_floats(const SelScanParams &p, bool grad)
{
    const Scratch s = scratch_of(p, form_of(p), grad);
    return s.chunks + s.shares + s.bc;
}

hipError_t launch_sel_scan(const SelScanParams &p, hipStream_t s)
{
    const Form f = form_of(p);
    if (!sel_scan_fits(p, false) || (f.chunks > 1 && !p.part) || p.gated != (p.z != nullptr) || p.keeps != (p.keep != nullptr)) return hipErrorInvalidValue;
    if (p.T == 1 && !p.states) {
        if (!p.y || !p.hT) return hipErrorInvalidValue;
        return p.dtype == DT_BF16 ? go_step<uint16_t>(p, f.L, s) : go_step<float>(p, f.L, s);
    }
    return p.dtype == DT_BF16 ? go<uint16_t>(false, p, f, s) : go<float>(false, p, f, s);
}

hipError_t launch_sel_scan_grad(const SelScanParams &p, hipStream_t s)
{
    if (!sel_scan_fits(p, true) || !p.part || !p.states || p.gated != (p.z != nullptr) || p.keeps != (p.keep != nullptr)) return hipErrorInvalidValue;
    const Form f = form_of(p);
    return p.dtype == DT_BF16 ? go<uint16_t>(true, p, f, s) : go<float>(true, p, f, s);
}

}  // namespace rl

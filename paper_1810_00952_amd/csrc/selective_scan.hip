// Selective state-space scan: every channel d has N numbers of state, and every token its own gates,
//
//   s = softplus(dt[t,d]),   h_t[d,n] = exp(s a[d,n]) h_(t-1)[d,n] + s x[t,d] B[t,n],   y[t,d] = (sum_n C[t,n] h_t[d,n] + skip[d] x[t,d]) z sigmoid(z)
//
// and its gradient, with du = dy z sigmoid(z): G_t[d,n] = C[t,n] du[t,d] + exp(s_(t+1) a) G_(t+1),
//   dB[t,n] = sum_d G s x,  dC[t,n] = sum_d du h,  dx = skip du + s sum_n G B,  da = sum_t G h_(t-1) exp(s a) s,
//   ds = sum_n G (h_(t-1) exp(s a) a + x B),  ddt = ds sigmoid(dt).
//
// A channel is four lanes', R of its states each (N <= 4 R), a wave sixteen channels', a workgroup of four waves sixty-four channels', which it walks by
// tiles of rows.  Of every four rows each of a channel's lanes finds what the channel needs once a token (softplus, the gate, products) for one and passes
// it to the other three as it is used, a lane move within the instruction that reads it; the sums over states go the other way, so that each
// lane ends with one row's.  B and C meet the lanes in LDS.  The sums over channels (dB, dC) halve the values a lane has with every step, by exchanges of the
// wave's halves and rows; the waves' meet in LDS, the workgroups' in memory, where another launch adds them up in a fixed order.  A row that is
// padding has s = s x = B = C = du = 0 and leaves state and derivative as they are.  Few channels: the rows are cut into chunks, a workgroup
// each; a launch ahead finds what each chunk makes of the state before it (P h + H; the derivative alike), P = exp(a sum s) as its fourth root, and the workgroups
// add up the chunks before theirs.
//
// The vector units bound it: a state and token is an exponential (four issue slots of a wave) and four more operations forwards, some twenty both ways.
// 8 x 2048 x 2048 x 16 bf16: forward 215 us, 57 % of them vector instructions of its one wave a SIMD, gradient 590, 67 %; two waves a SIMD of
// the gradient would spill (656 -> 1690).  1 x 16384 x 2048 x 16 in documents: 148 of the launch ahead and 179, 77 % by two waves.  One token of 64 sequences: 7 us.
#include <algorithm>
#include <type_traits>

#include "igemm_lds.h"

namespace rl {

namespace {

constexpr int LANES = 4, CHANNELS = 64;       // lanes of a channel, channels of a workgroup
constexpr float LOG2E = 1.4426950408889634f;

// Rows of a tile: of the gradient as many as its states and gates fit the registers; 32 forwards gave nothing
constexpr int rows_of(int R) { return R <= 4 ? 16 : 64 / R; }

// A chunk makes P h + H of the state h before it.  P h is a number of f32 where P = exp(a sum s) is none: of a state that grows what was small before, or
// zero.  So P is there as its fourth root, between 2^-126 and 2^127, which takes an h of any size to zero or infinity, but zero and infinity to themselves.
// -0, which is no such root, where a document's first row is part of the chunk.
constexpr float FIRST = -0.0f;
__device__ __forceinline__ bool is_first(float root) { return __float_as_uint(root) == 0x80000000u; }
__device__ __forceinline__ float through(float root, float h, float H)
{
    const float y = __builtin_fmaf(h * root * root * root, root, H);
    return is_first(root) ? H : y;
}
__device__ __forceinline__ float exp2_(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(v);
#else
    return v;
#endif
}

// An infinite number as the largest finite one, NaN as it is.  Rows that are no tokens hold a state as such of step 0, and 0 times a has to be 0 in them; a token's
// exp(s a) is the same number.
__device__ __forceinline__ float finite_(float v) { return fabsf(v) == INFINITY ? copysignf(3.402823466e38f, v) : v; }

// the fourth root of 2^v
__device__ __forceinline__ float root_of(float v) { return exp2_(fminf(fmaxf(0.25f * v, -126.0f), 127.0f)); }

__device__ __forceinline__ float log2_(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_logf(v);
#else
    return v;
#endif
}

// s = ln(1 + e^v) and its slope, sigmoid(v).  With w = e^v: ln of 1 + w as it is rounded, and what the rounding took off w, whose part of the logarithm
// is itself where 1 + w is below 2, and above it less than the logarithm's last bit.  For v above 20 it is v, as rounded.
__device__ __forceinline__ float softplus(float v, float &slope)
{
    const float w = exp2_(v * LOG2E), u = 1.0f + w, lost = w - (u - 1.0f);
    const float s = __builtin_fmaf(log2_(u), 0.6931471805599453f, u < 2.0f ? lost : 0.0f);
    slope = v > 20.0f ? 1.0f : w * rcp_(u);
    return v > 20.0f ? v : s;
}
__device__ __forceinline__ float softplus(float v)
{
    float slope;
    return softplus(v, slope);
}

template <typename E> struct Bits;
template <> struct Bits<float> { typedef uint32_t raw; };
template <> struct Bits<uint16_t> { typedef uint16_t raw; };
template <typename E> __device__ __forceinline__ float number(typename Bits<E>::raw r)
{
    if constexpr (sizeof(E) == 4) return __uint_as_float(r);
    else return bf16_bits_to_f32(r);
}
template <typename E> __device__ __forceinline__ float at(const void *p, int64_t i) { return number<E>(((const typename Bits<E>::raw *)p)[i]); }
template <typename E> __device__ __forceinline__ void put(void *p, int64_t i, float v)
{
    if constexpr (sizeof(E) == 4) ((float *)p)[i] = v;
    else ((uint16_t *)p)[i] = (uint16_t)pack_bf16x2(v, v);
}

template <int CTRL> __device__ __forceinline__ float moved(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
#else
    return v;
#endif
}
// lane k's of the channel's four
template <int K> __device__ __forceinline__ float of_lane(float v) { return moved<K * 0x55>(v); }
// four numbers of every lane summed over the channel's lanes: lane l gets the sum of number l
__device__ __forceinline__ float over_states(const float (&v)[4])
{
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    const float a = (odd ? v[1] : v[0]) + moved<0xb1>(odd ? v[0] : v[1]), b = (odd ? v[3] : v[2]) + moved<0xb1>(odd ? v[2] : v[3]);
    return (high ? b : a) + moved<0x4e>(high ? a : b);
}
// a in the lower half, b in the upper half of the wave (ROWS: in even and odd rows of sixteen lanes), each summed over both
template <bool ROWS> __device__ __forceinline__ float halves(float a, float b)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = ROWS ? __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false)
                        : __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
#else
    return a + b;
#endif
}
// R numbers each of dB and dC summed over a wave's channels.  Number r of B (C) and of a channel's lane l is at i = r / 4, in lane
// slot_of(which, r, l); lanes with bit 2 hold nothing of use.
constexpr int sums_of(int R) { return R > 4 ? R / 4 : 1; }
__device__ __forceinline__ int slot_of(int which, int r, int l) { return which * 32 + (r & 1) * 16 + (r >> 1 & 1) * 8 + l; }
template <int R> __device__ __forceinline__ void over_channels(const float (&db)[R], const float (&dc)[R], float (&out)[sums_of(R)])
{
    float w[R], u[R > 1 ? R / 2 : 1];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = halves<false>(db[r], dc[r]);
#pragma unroll
    for (int r = 0; r < (R > 1 ? R / 2 : 1); ++r) u[r] = halves<true>(w[2 * r < R ? 2 * r : 0], w[2 * r + 1 < R ? 2 * r + 1 : 0]);
    const bool high = threadIdx.x & 8;
#pragma unroll
    for (int i = 0; i < sums_of(R); ++i) {
        float v;
        if constexpr (R >= 4) v = (high ? u[2 * i + 1] : u[2 * i]) + moved<0x128>(high ? u[2 * i] : u[2 * i + 1]);      // row_ror 8
        else v = u[0] + moved<0x128>(u[0]);
        out[i] = v + moved<0x104>(v);                                                                             // row_shl 4
    }
}

// Barrier of a workgroup whose waves meet in LDS alone: what is under way to and from memory stays so
__device__ __forceinline__ void lds_barrier()
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#endif
}

// what a lane works on
template <int R>
struct Place {
    int l;                                    // its states l R ..; of every four rows the l-th
    int64_t b, d;
    int32_t chunk, slab;
    bool live;
    __device__ __forceinline__ Place(const SelScanParams &p, int32_t slabs, int32_t first_chunk = 0)
    {
        l = threadIdx.x & 3;
        const uint32_t rest = blockIdx.x / (uint32_t)slabs;
        slab = (int32_t)(blockIdx.x - rest * slabs);
        chunk = (int32_t)(rest / (uint32_t)p.B);
        b = rest - (uint32_t)chunk * (uint32_t)p.B;
        chunk += first_chunk;
        d = (int64_t)slab * CHANNELS + (threadIdx.x >> 2);
        live = d < p.D;
        if (!live) d = 0;                     // some other channel's, of which nothing is stored
    }
    // R numbers of a [D][N] matrix, zeros for the states behind N
    __device__ __forceinline__ void load(const SelScanParams &p, const float *m, float (&v)[R]) const
    {
        const float *q = m + d * p.N + l * R;
        if (R % 4 == 0 && p.N == LANES * R) {
#pragma unroll
            for (int r = 0; r < R; r += 4) {
                const f32x4 t = *(const f32x4 *)(q + (r < R ? r : 0));
#pragma unroll
                for (int k = 0; k < 4 && k < R; ++k) v[r + k < R ? r + k : 0] = t[k];
            }
            return;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = l * R + r < p.N ? q[r] : 0.0f;
    }
    __device__ __forceinline__ void store(const SelScanParams &p, float *m, const float (&v)[R]) const
    {
        if (!live) return;
        float *q = m + d * p.N + l * R;
        if (R % 4 == 0 && p.N == LANES * R) {
#pragma unroll
            for (int r = 0; r + 3 < R; r += 4) *(f32x4 *)(q + r) = f32x4{v[r], v[r + 1 < R ? r + 1 : r], v[r + 2 < R ? r + 2 : r], v[r + 3 < R ? r + 3 : r]};
            return;
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (l * R + r < p.N) q[r] = v[r];
    }
};

// floats from one share of da and dskip to the next: whole vectors, by which da goes
__host__ __device__ __forceinline__ int64_t share_floats(const SelScanParams &p) { return (p.D * p.N + p.D + 3) / 4 * 4; }

// rows of a tile that are tokens, that are a document's first; their flags are asked for a tile before
template <bool KEEP, int ROWS> struct Flags {
    uint32_t tok, first;
    int asked;
    int64_t left;
    __device__ __forceinline__ void request(const SelScanParams &p, int64_t b, int64_t t0)
    {
        left = p.T - t0;
        const int i = threadIdx.x & 63;
        if (KEEP) asked = i < ROWS && i < left ? p.keep[b * p.T + t0 + i] : 0;
    }
    __device__ __forceinline__ void look()
    {
        if (KEEP) {
            tok = (uint32_t)__ballot(asked != 0);
            first = (uint32_t)__ballot(asked == 2);
        } else {
            tok = left >= ROWS ? ~0u : (1u << (left > 0 ? left : 0)) - 1u;
            first = 0;
        }
    }
};

// rows in memory: `room` bytes from a tile's first row to the sequence's last.  What lies behind them reads as zero and is not written; so
// does what a lane without a channel or state (offset OOB) asks for.
__device__ __forceinline__ rsrc_t rows_at(const void *first, int64_t room)
{
    return make_rsrc(first, (uint32_t)(room < 0x7fffffff ? room : 0x7fffffff));
}
template <typename E> __device__ __forceinline__ typename Bits<E>::raw fetch(const rsrc_t &r, uint32_t off, uint32_t more)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(E) == 4) return __builtin_amdgcn_raw_buffer_load_b32(r, off, more, 0);
    else return __builtin_amdgcn_raw_buffer_load_b16(r, off, more, 0);
#else
    return 0;
#endif
}
template <typename E> __device__ __forceinline__ void put(const rsrc_t &r, uint32_t off, uint32_t more, float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, off, more, 0);
    else __builtin_amdgcn_raw_buffer_store_b16((uint16_t)pack_bf16x2(v, v), r, off, more, 0);
#endif
}

// B and C of a tile's rows on their way to LDS, to the wave's own part of it: zeros behind N and of padding.  Where N is all of the lanes' states the rows
// of a tile lie in memory as they do there, and go by whole vectors.
template <typename E, int R, int ROWS> struct Stage {
    static constexpr int WIDE = LANES * R, TOTAL = 2 * ROWS * WIDE, EACH = TOTAL / 64, KV = 16 / sizeof(E), VECS = TOTAL / KV, EACHV = (VECS + 63) / 64;
    typename Bits<E>::raw r[EACH];
    u32x4 v[EACHV];
    rsrc_t rows;
    uint32_t off[EACH], line;
    bool whole;
    __device__ __forceinline__ Stage(const SelScanParams &p, int64_t row0, int64_t left)
    {
        line = (uint32_t)(2 * p.N * sizeof(E));
        rows = rows_at((const char *)p.bc + row0 * line, left * line);
        whole = p.N == WIDE;
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = e * 64 + lane, n = i % WIDE, which = i / WIDE % 2, t = i / (2 * WIDE);
            off[e] = n < p.N ? (uint32_t)((t * 2 + which) * (int)p.N + n) * (uint32_t)sizeof(E) : OOB;
        }
    }
    __device__ __forceinline__ void request(uint32_t t0)                       // rows from the first of them
    {
#if defined(__HIP_DEVICE_COMPILE__)
        const uint32_t from = t0 * line;
        if (whole) {
#pragma unroll
            for (int e = 0; e < EACHV; ++e) v[e] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, from + (e * 64 + (threadIdx.x & 63)) * 16, 0, 0));
        } else {
#pragma unroll
            for (int e = 0; e < EACH; ++e) r[e] = fetch<E>(rows, off[e], from);
        }
#endif
    }
    __device__ __forceinline__ void put(float *s, uint32_t tok) const
    {
        const int lane = threadIdx.x & 63;
        if (whole) {
#pragma unroll
            for (int e = 0; e < EACHV; ++e) {
                const int i = (e * 64 + lane) * KV;
                if (VECS % 64 != 0 && i >= TOTAL) break;
                const bool here = tok >> (i / (2 * WIDE)) & 1;
#pragma unroll
                for (int k = 0; k < KV; k += 4) {
                    f32x4 q;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if constexpr (sizeof(E) == 4) q[c] = __uint_as_float(v[e][c]);
                        else q[c] = __uint_as_float(c & 1 ? v[e][(k + c) / 2] & 0xffff0000u : v[e][(k + c) / 2] << 16);
                        if (!here) q[c] = 0.0f;
                    }
                    *(f32x4 *)(s + i + k) = q;
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int i = e * 64 + lane;
                s[i] = tok >> (i / (2 * WIDE)) & 1 ? number<E>(r[e]) : 0.0f;
            }
        }
    }
};

// a row's R numbers of B or C
template <int R> __device__ __forceinline__ void from_lds(const float *s, float (&v)[R])
{
    if constexpr (R >= 4) {
#pragma unroll
        for (int r = 0; r < R; r += 4) {
            const f32x4 t = *(const f32x4 *)(s + r);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[r + k] = t[k];
        }
    } else if constexpr (R == 2) {
        const f32x2 t = *(const f32x2 *)s;
        v[0] = t[0]; v[1] = t[1];
    } else {
        v[0] = s[0];
    }
}

// B and C of the rows to come, read AHEAD rows before they are used, across the tiles: the compiler, which counts on more waves than there are, would
// read them where they are used.  Row k of a walk through a tile; from ROWS on the next tile's, which lies in the other half of the wave's LDS.
template <int R, int ROWS, bool BACK, bool WITH_B, bool WITH_C> struct Coming {
    static constexpr int AHEAD = R >= 16 ? 1 : R >= 4 ? 2 : 4, RING = 2 * AHEAD;
    static_assert(ROWS % RING == 0, "a tile's first row is in the ring's first place");
    float b[RING][R], c[RING][R];
    const float *s;                            // the lane's part of the two halves
    __device__ __forceinline__ void read(int k, int half)
    {
        const int t = BACK ? ROWS - 1 - k % ROWS : k % ROWS;
        const float *q = s + (half * ROWS + t) * 2 * LANES * R;
        if (WITH_B) from_lds<R>(q, b[k % RING]);
        if (WITH_C) from_lds<R>(q + LANES * R, c[k % RING]);
    }
    __device__ __forceinline__ void start(const float *s_, int half)
    {
        s = s_;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) read(k, half);
    }
    // row k of the tile in `half` is next
    __device__ __forceinline__ void step(int k, int half)
    {
        read(k + AHEAD, k + AHEAD < ROWS ? half : half ^ 1);
#if defined(__HIP_DEVICE_COMPILE__)
        __builtin_amdgcn_sched_barrier(0x47f);        // all but accesses of LDS may cross
#endif
    }
    __device__ __forceinline__ float B(int k, int r) const { return b[k % RING][r]; }
    __device__ __forceinline__ float C(int k, int r) const { return c[k % RING][r]; }
};

// a lane's rows of a tile, the l-th of every four: `off` bytes from the tile's first, four rows on from one to the next
template <typename E, int ROWS> struct Column {
    typename Bits<E>::raw r[ROWS / 4];
    __device__ __forceinline__ void request(const rsrc_t &rows, uint32_t off, uint32_t line)
    {
#pragma unroll
        for (int i = 0; i < ROWS / 4; ++i) r[i] = fetch<E>(rows, off, 4 * i * line);
    }
};

}  // namespace

// ---------------------------------------------------------------------------
// one token a sequence
// ---------------------------------------------------------------------------
template <typename E, int R>
__global__ __launch_bounds__(256) void selective_scan_step_kernel(const SelScanParams p, int32_t slabs)
{
    const Place<R> at_(p, slabs);
    const int64_t DN = p.D * p.N, c = at_.b * p.D + at_.d;
    const int flag = p.keep ? p.keep[at_.b] : 1;
    float a[R], h[R], B[R], C[R];
    at_.load(p, p.h0 + at_.b * DN, h);
    at_.load(p, p.a, a);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int n = at_.l * R + r;
        B[r] = n < p.N ? at<E>(p.bc, at_.b * 2 * p.N + n) : 0.0f;
        C[r] = n < p.N ? at<E>(p.bc, (at_.b * 2 + 1) * p.N + n) : 0.0f;
    }
    const float x = at<E>(p.x, c), s = softplus(at<E>(p.dt, c)), v = s * x, skip = p.skip[at_.d], z = p.z ? at<E>(p.z, c) : 0.0f;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (flag) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float e = exp2_(s * finite_(a[r] * LOG2E));
            h[r] = __builtin_fmaf(e, flag == 2 ? 0.0f : h[r], v * B[r]);
            sum[0] = __builtin_fmaf(C[r], h[r], sum[0]);
        }
    }
    at_.store(p, p.hT + at_.b * DN, h);
    float y = __builtin_fmaf(skip, x, over_states(sum));
    if (p.z) y *= z * sigmoidf_(z);
    if (at_.l == 0 && at_.live) put<E>(p.y, c, flag ? y : 0.0f);
}

// ---------------------------------------------------------------------------
// forward.  AHEAD: what a chunk makes of the state before it, into part ([chunk][b] P's root, H of [D][N])
// ---------------------------------------------------------------------------
template <typename E, int R, bool KEEP, bool GATED, bool AHEAD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 4))) void selective_scan_kernel(const SelScanParams p, int32_t slabs, int32_t chunks, int32_t chunk_rows)
{
    constexpr int ROWS = rows_of(R);
    const Place<R> at_(p, slabs);
    const int64_t DN = p.D * p.N;
    const int l = at_.l;
    __shared__ __attribute__((aligned(16))) float sb[4][2][ROWS][2][LANES * R];          // of every wave
    float a2[R], h[R], total = 0.0f;
    at_.load(p, p.a, a2);
#pragma unroll
    for (int r = 0; r < R; ++r) { a2[r] = finite_(a2[r] * LOG2E); h[r] = 0.0f; }
    bool began = false;                                              // a document's first row was there
    if (!AHEAD) {
        at_.load(p, p.h0 + at_.b * DN, h);
#pragma unroll 8
        for (int32_t k = 0; k < at_.chunk; ++k) {
            float f[R], H[R];
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b)) * DN, f);
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b) + 1) * DN, H);
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = through(f[r], h[r], H[r]);
        }
    }
    const float skip = p.skip[at_.d];
    const int64_t T0 = (int64_t)at_.chunk * chunk_rows, row0 = at_.b * p.T + T0, left = min(p.T - T0, (int64_t)chunk_rows);
    const int32_t tiles = (int32_t)((left + ROWS - 1) / ROWS);
    const uint32_t line = (uint32_t)(p.D * sizeof(E));
    auto rows = [&](const void *x) { return rows_at((const char *)x + row0 * line, x ? left * line : 0); };      // the chunk's
    const rsrc_t from_x = rows(p.x), from_t = rows(p.dt), from_z = rows(p.z), to = rows(p.y);
    uint32_t off = at_.live ? l * line + (uint32_t)(at_.d * sizeof(E)) : OOB, ask = off;
    const uint32_t on = at_.live ? ROWS * line : 0;                  // a tile on
    Column<E, ROWS> qx, qt, qz;
    Stage<E, R, ROWS> bc(p, row0, left);
    auto request = [&](int32_t tile) {
        bc.request((uint32_t)tile * ROWS);
        qx.request(from_x, ask, line);
        qt.request(from_t, ask, line);
        if (GATED && !AHEAD) qz.request(from_z, ask, line);
        ask += on;
    };
    // what the rows need once a token is found before the tile they are of begins: with few waves nothing else hides how long that takes
    float x[ROWS / 4], s[ROWS / 4], z[ROWS / 4], nx[ROWS / 4], ns[ROWS / 4], nz[ROWS / 4];
    uint32_t tok, first;
    Flags<KEEP, ROWS> next;
    auto once = [&]() {
#pragma unroll
        for (int i = 0; i < ROWS / 4; ++i) {
            const bool here = next.tok >> (4 * i + l) & 1;
            const float step = softplus(number<E>(qt.r[i]));
            nx[i] = here ? number<E>(qx.r[i]) : 0.0f;
            ns[i] = here ? step : 0.0f;
            nz[i] = GATED && !AHEAD ? number<E>(qz.r[i]) : 0.0f;
            if (GATED && !AHEAD) nz[i] *= sigmoidf_(nz[i]);
        }
    };
    auto turn = [&]() {
        tok = next.tok;
        first = next.first;
#pragma unroll
        for (int i = 0; i < ROWS / 4; ++i) { x[i] = nx[i]; s[i] = ns[i]; z[i] = nz[i]; }
    };
    float *const mine = &sb[threadIdx.x >> 6][0][0][0][0];
    constexpr int HALF = ROWS * 2 * LANES * R;
    request(0);
    next.request(p, at_.b, T0);
    next.look();
    bc.put(mine, next.tok);
    once();
    turn();
    wave_lds_exchange();
    Coming<R, ROWS, false, true, !AHEAD> bcs;
    bcs.start(mine + l * R, 0);
    float *state = p.states ? p.states + (at_.b * ((p.T + ROWS - 1) / ROWS) + T0 / ROWS) * DN : nullptr;
    for (int32_t tile = 0; tile < tiles; ++tile) {
        const int half = tile & 1;
        request(tile + 1);                                           // behind the chunk: zeros
        next.request(p, at_.b, T0 + (int64_t)(tile + 1) * ROWS);
        if (!AHEAD && state) {
            at_.store(p, state, h);
            state += DN;
        }
        // with a document's first row among them, whose states are masked row by row, and without
        auto walk = [&](auto masked) {
#pragma unroll
            for (int i = 0; i < ROWS / 4; ++i) {
                float sum[4];
                const float v = s[i] * x[i];
                if (AHEAD) total += s[i];
                if (i + 1 == ROWS / 4) {
                    next.look();
                    bc.put(mine + (half ^ 1) * HALF, next.tok);
                    once();
                    wave_lds_exchange();
                }
                auto row = [&](auto lane) {
                    constexpr int K = decltype(lane)::value;
                    const int t = 4 * i + K;
                    bcs.step(t, half);
                    if (masked && (first >> t & 1)) {
#pragma unroll
                        for (int r = 0; r < R; ++r) h[r] = 0.0f;
                    }
                    sum[K] = 0.0f;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        h[r] = __builtin_fmaf(exp2_(of_lane<K>(s[i]) * a2[r]), h[r], of_lane<K>(v) * bcs.B(t, r));
                        if (!AHEAD) sum[K] = __builtin_fmaf(bcs.C(t, r), h[r], sum[K]);
                    }
                };
                row(std::integral_constant<int, 0>{});
                row(std::integral_constant<int, 1>{});
                row(std::integral_constant<int, 2>{});
                row(std::integral_constant<int, 3>{});
                if (!AHEAD) {
                    float y = __builtin_fmaf(skip, x[i], over_states(sum));
                    if (GATED) y *= z[i];
                    put<E>(to, off, 4 * i * line, !KEEP || (tok >> (4 * i + l) & 1) ? y : 0.0f);
                }
            }
        };
        if (KEEP && first) {
            began = true;
            walk(std::true_type{});
        } else {
            walk(std::false_type{});
        }
        off += on;
        turn();
    }
    if (AHEAD) {
        total += moved<0xb1>(total);                                 // of a channel's four lanes
        total += moved<0x4e>(total);
        float f[R];
#pragma unroll
        for (int r = 0; r < R; ++r) f[r] = began ? FIRST : root_of(total * a2[r]);
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b)) * DN, f);
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b) + 1) * DN, h);
    } else if (p.hT && at_.chunk + 1 == chunks) {
        at_.store(p, p.hT + at_.b * DN, h);
    }
}

// ---------------------------------------------------------------------------
// gradient, tiles from the last to the first.  AHEAD: what a chunk makes of the derivative behind it, into part
// ---------------------------------------------------------------------------
template <typename E, int R, bool KEEP, bool GATED, bool AHEAD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, AHEAD ? 4 : 2))) void selective_scan_grad_kernel(const SelScanParams p, int32_t slabs, int32_t chunks, int32_t chunk_rows, float *shares, float *bc_shares)
{
    constexpr int ROWS = rows_of(R), SUMS = sums_of(R);
    constexpr uint32_t FULL = (1u << ROWS) - 1u;
    const Place<R> at_(p, slabs, AHEAD ? 1 : 0);
    const int64_t DN = p.D * p.N;
    const int l = at_.l, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __shared__ __attribute__((aligned(16))) float sb[4][2][ROWS][2][LANES * R];          // of every wave
    __shared__ float sc[AHEAD ? 1 : 2][4][ROWS][SUMS][64];           // dB, dC of a wave's channels
    float a[R], a2[R], G[R], da[R], total = 0.0f, dskip = 0.0f;
    at_.load(p, p.a, a);
#pragma unroll
    for (int r = 0; r < R; ++r) { a[r] = finite_(a[r]); a2[r] = finite_(a[r] * LOG2E); G[r] = 0.0f; da[r] = 0.0f; }
    bool began = false;
    if (!AHEAD) {
        at_.load(p, p.dhT + at_.b * DN, G);
#pragma unroll 8
        for (int32_t k = chunks - 1; k > at_.chunk; --k) {
            float f[R], H[R];
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b)) * DN, f);
            at_.load(p, p.part + (2 * ((int64_t)k * p.B + at_.b) + 1) * DN, H);
#pragma unroll
            for (int r = 0; r < R; ++r) G[r] = through(f[r], G[r], H[r]);
        }
    }
    const float skip = p.skip[at_.d];
    const int64_t T0 = (int64_t)at_.chunk * chunk_rows, row0 = at_.b * p.T + T0, left = min(p.T - T0, (int64_t)chunk_rows);
    const int32_t tiles = (int32_t)((left + ROWS - 1) / ROWS);
    const uint32_t line = (uint32_t)(p.D * sizeof(E));
    auto rows = [&](const void *x) { return rows_at((const char *)x + row0 * line, x ? left * line : 0); };      // the chunk's
    const rsrc_t from_x = rows(p.x), from_t = rows(p.dt), from_d = rows(p.dy), from_z = rows(p.z), to_x = rows(p.dx), to_t = rows(p.ddt), to_z = rows(p.dz);
    const uint32_t on = at_.live ? ROWS * line : 0;                  // a tile on
    uint32_t off = (at_.live ? l * line + (uint32_t)(at_.d * sizeof(E)) : OOB) + (uint32_t)(tiles - 1) * on, ask = off;
    Column<E, ROWS> qx, qt, qd, qz;
    Stage<E, R, ROWS> bc(p, row0, left);
    float h[R], next_h[R];
    const float *state = p.states + (at_.b * ((p.T + ROWS - 1) / ROWS) + T0 / ROWS + tiles - 1) * DN;
    auto request = [&](int32_t tile) {
        bc.request((uint32_t)tile * ROWS);
        if (!AHEAD) qx.request(from_x, ask, line);
        qt.request(from_t, ask, line);
        qd.request(from_d, ask, line);
        if (GATED) qz.request(from_z, ask, line);
        if (!AHEAD) at_.load(p, state, next_h);
        ask -= on;
        state -= DN;
    };
    // once a token, a tile ahead.  dz: dy times the gate's slope
    float x[ROWS / 4], s[ROWS / 4], slope[ROWS / 4], du[ROWS / 4], dz[ROWS / 4], nx[ROWS / 4], ns[ROWS / 4], nslope[ROWS / 4], ndu[ROWS / 4], ndz[ROWS / 4];
    uint32_t tok, first;
    Flags<KEEP, ROWS> next;
    auto once = [&]() {
#pragma unroll
        for (int i = 0; i < ROWS / 4; ++i) {
            const bool here = at_.live && (next.tok >> (4 * i + l) & 1);     // channels that are not there add nothing to dB and dC
            const float step = softplus(number<E>(qt.r[i]), nslope[i]), dy = here ? number<E>(qd.r[i]) : 0.0f, z = GATED && here ? number<E>(qz.r[i]) : 0.0f;
            nx[i] = !AHEAD && here ? number<E>(qx.r[i]) : 0.0f;
            ns[i] = here ? step : 0.0f;
            const float sg = GATED ? sigmoidf_(z) : 0.0f;
            ndu[i] = GATED ? dy * (z * sg) : dy;
            ndz[i] = GATED && !AHEAD ? dy * __builtin_fmaf(z * sg, sigmoidf_(-z), sg) : 0.0f;
        }
    };
    auto turn = [&]() {
        tok = next.tok;
        first = next.first;
#pragma unroll
        for (int i = 0; i < ROWS / 4; ++i) {
            x[i] = nx[i]; s[i] = ns[i]; slope[i] = nslope[i]; du[i] = ndu[i]; dz[i] = ndz[i];
        }
        if (!AHEAD) {
#pragma unroll
            for (int r = 0; r < R; ++r) h[r] = next_h[r];
        }
    };
    float *const mine = &sb[wave][0][0][0][0];
    constexpr int HALF = ROWS * 2 * LANES * R;
    request(tiles - 1);
    next.request(p, at_.b, T0 + (int64_t)(tiles - 1) * ROWS);
    next.look();
    bc.put(mine + ((tiles - 1) & 1) * HALF, next.tok);
    once();
    turn();
    wave_lds_exchange();
    Coming<R, ROWS, AHEAD, !AHEAD, GATED || AHEAD> fore;             // of the first way through a tile
    fore.start(mine + l * R, (tiles - 1) & 1);
    for (int32_t tile = tiles - 1; tile >= 0; --tile) {
        const int half = tile & 1;
        // in front of the chunk: what is asked for again is not used
        if (tile > 0) {
            request(tile - 1);
            next.request(p, at_.b, T0 + (int64_t)(tile - 1) * ROWS);
        }
        auto stage = [&]() {
            next.look();
            bc.put(mine + (half ^ 1) * HALF, next.tok);
            once();
            wave_lds_exchange();
        };
        if constexpr (AHEAD) {
#pragma unroll
            for (int i = ROWS / 4 - 1; i >= 0; --i) {
                total += s[i];
                if (i == 0) stage();
                auto row = [&](auto lane_) {
                    constexpr int K = decltype(lane_)::value;
                    const int t = 4 * i + K;
                    fore.step(ROWS - 1 - t, half);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        G[r] = __builtin_fmaf(fore.C(ROWS - 1 - t, r), of_lane<K>(du[i]), G[r]) * exp2_(of_lane<K>(s[i]) * a2[r]);
                        if (KEEP && (first >> t & 1)) G[r] = 0.0f;
                    }
                };
                row(std::integral_constant<int, 3>{});
                row(std::integral_constant<int, 2>{});
                row(std::integral_constant<int, 1>{});
                row(std::integral_constant<int, 0>{});
            }
            began |= KEEP && first != 0;
        } else {
            // with padding, rows behind the sequence's last or a document's first row among them, and without
            auto walk = [&](auto masked) {
                float decayed[ROWS][R], gate[ROWS][R], u[ROWS / 4], dat[R];       // the state before a row times its gate
                Coming<R, ROWS, true, true, true> back;
#pragma unroll
                for (int i = 0; i < ROWS / 4; ++i) {
                    float sum[4];
                    const float v = s[i] * x[i];
                    if (i + 1 == ROWS / 4) back.start(mine + l * R, half);
                    auto row = [&](auto lane_) {
                        constexpr int K = decltype(lane_)::value;
                        const int t = 4 * i + K;
                        if (t + fore.AHEAD < ROWS) fore.step(t, half);
                        if (masked && (first >> t & 1)) {
#pragma unroll
                            for (int r = 0; r < R; ++r) h[r] = 0.0f;
                        }
                        sum[K] = 0.0f;
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            gate[t][r] = exp2_(of_lane<K>(s[i]) * a2[r]);
                            decayed[t][r] = gate[t][r] * h[r];
                            h[r] = __builtin_fmaf(of_lane<K>(v), fore.B(t, r), decayed[t][r]);
                            if (GATED) sum[K] = __builtin_fmaf(fore.C(t, r), h[r], sum[K]);
                        }
                    };
                    row(std::integral_constant<int, 0>{});
                    row(std::integral_constant<int, 1>{});
                    row(std::integral_constant<int, 2>{});
                    row(std::integral_constant<int, 3>{});
                    u[i] = GATED ? __builtin_fmaf(skip, x[i], over_states(sum)) : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < R; ++r) dat[r] = 0.0f;
#pragma unroll
                for (int i = ROWS / 4 - 1; i >= 0; --i) {
                    const float v = s[i] * x[i];
                    float gb[4], ga[4];
                    if (i == 0) stage();
                    auto row = [&](auto lane_) {
                        constexpr int K = decltype(lane_)::value;
                        const int t = 4 * i + K;
                        float db[R], dc[R], out[SUMS];
                        if (ROWS - 1 - t + back.AHEAD < ROWS) back.step(ROWS - 1 - t, half);
                        gb[K] = 0.0f;
                        ga[K] = 0.0f;
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const float he = decayed[t][r], B = back.B(ROWS - 1 - t, r);
                            G[r] = __builtin_fmaf(back.C(ROWS - 1 - t, r), of_lane<K>(du[i]), G[r]);
                            // in the sum over rows a state and a derivative that padding holds, were they infinite or NaN, are none; its other results are masked as they leave
                            const float arg = masked && !(tok >> t & 1) ? 0.0f : G[r] * he;
                            dat[r] = __builtin_fmaf(of_lane<K>(s[i]), arg, dat[r]);
                            ga[K] = __builtin_fmaf(arg, a[r], ga[K]);
                            gb[K] = __builtin_fmaf(G[r], B, gb[K]);
                            db[r] = of_lane<K>(v) * G[r];
                            dc[r] = of_lane<K>(du[i]) * __builtin_fmaf(of_lane<K>(v), B, he);
                            G[r] *= gate[t][r];
                            if (masked && (first >> t & 1)) G[r] = 0.0f;
                        }
                        over_channels<R>(db, dc, out);
#pragma unroll
                        for (int k = 0; k < SUMS; ++k) sc[half][wave][t][k][lane] = out[k];
                    };
                    row(std::integral_constant<int, 3>{});
                    row(std::integral_constant<int, 2>{});
                    row(std::integral_constant<int, 1>{});
                    row(std::integral_constant<int, 0>{});
                    const float sgb = over_states(gb), sga = over_states(ga);
                    dskip = __builtin_fmaf(du[i], x[i], dskip);
                    const bool here = !masked || (tok >> (4 * i + l) & 1);
                    put<E>(to_x, off, 4 * i * line, here ? __builtin_fmaf(skip, du[i], s[i] * sgb) : 0.0f);
                    put<E>(to_t, off, 4 * i * line, here ? __builtin_fmaf(x[i], sgb, sga) * slope[i] : 0.0f);
                    if (GATED) put<E>(to_z, off, 4 * i * line, here ? dz[i] * u[i] : 0.0f);
                }
#pragma unroll
                for (int r = 0; r < R; ++r) da[r] += dat[r];             // tile by tile: fewer roundings on the way
            };
            if ((KEEP && first) || (tok & FULL) != FULL) walk(std::true_type{});
            else walk(std::false_type{});
            fore.start(mine + l * R, half ^ 1);
            lds_barrier();
            const int32_t t0 = tile * ROWS;
            constexpr int WIDE = LANES * R;
#pragma unroll
            for (int e = 0; e < (ROWS * 2 * WIDE + 255) / 256; ++e) {
                const int i = e * 256 + (int)threadIdx.x, n = i % WIDE, which = i / WIDE % 2, t = i / (2 * WIDE);
                if (t >= ROWS || n >= p.N || t0 + t >= left) continue;
                const int r = n % R, slot = slot_of(which, r, n / R);
                float sum = sc[half][0][t][r / 4][slot];
#pragma unroll
                for (int w = 1; w < 4; ++w) sum += sc[half][w][t][r / 4][slot];
                bc_shares[((int64_t)at_.slab * p.B * p.T + row0 + t0 + t) * 2 * p.N + which * p.N + n] = tok >> t & 1 ? sum : 0.0f;
            }
        }
        off -= on;
        turn();
    }
    if constexpr (AHEAD) {
        total += moved<0xb1>(total);
        total += moved<0x4e>(total);
        float f[R];
#pragma unroll
        for (int r = 0; r < R; ++r) f[r] = began ? FIRST : root_of(total * a2[r]);
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b)) * DN, f);
        at_.store(p, p.part + (2 * ((int64_t)at_.chunk * p.B + at_.b) + 1) * DN, G);
        return;
    }
    if (at_.chunk == 0) at_.store(p, p.dh0 + at_.b * DN, G);
    float *share = shares + ((int64_t)at_.chunk * p.B + at_.b) * share_floats(p);
    at_.store(p, share, da);
    dskip += moved<0xb1>(dskip);
    dskip += moved<0x4e>(dskip);
    if (at_.live && l == 0) share[DN + at_.d] = dskip;
}

namespace {

struct Form { int R; int32_t slabs, chunks, chunk_rows; };

// Chunks where there are fewer workgroups than CUs: of 64 rows and more, in whole tiles, as many as fill the CUs once with the
// gradient's workgroups, whose registers are a CU's, twice with the forward pass' (1 x 16384 x 2048 x 16 bf16 forward 431 -> 378 us; 3 x 777 x 515 x 24 f32
// gradient in 297 workgroups 91, in 243 61)
Form form_of(const SelScanParams &p, bool grad)
{
    Form f;
    f.R = 1;
    while (f.R * LANES < p.N) f.R *= 2;
    const int64_t rows = rows_of(f.R), tiles = (p.T + rows - 1) / rows;
    f.slabs = (int32_t)((p.D + CHANNELS - 1) / CHANNELS);
    const int64_t wgs = p.B * f.slabs, most = tiles * rows / 64;
    int64_t chunks = wgs < 256 ? (grad ? 256 : 512) / wgs : 1;
    if (chunks > most) chunks = most > 0 ? most : 1;
    // a chunk's rows against the chunks before it, which each workgroup adds up: some 0.3 us a row, 0.15 a chunk
    while (chunks * chunks > 2 * p.T) chunks -= chunks / 8 + 1;
    // not two forwards, whose launch ahead walks half of the rows once more and leaves the CUs as they were: 2048 rows of 16 states in 192 workgroups 230 us in two chunks, 196
    // in one, in 255 235 and 198, in 256 238 and 199 (64 states in 192: 949 and 668); in 160 three chunks take 184, one 195 (64 states 715 and 667); 128 rows in 32 workgroups 16.9 and 15.5.  The gradient's gain: in 128 two 534, one 725
    if (!grad && chunks < 3) chunks = 1;
    // a chunk's rows are reached by 31-bit offsets
    const int64_t line = std::max(p.D, 2 * p.N) * (p.dtype == DT_BF16 ? 2 : 4), reach = ((int64_t)1 << 30) / (line * rows);
    if (chunks < (tiles + reach - 1) / reach) chunks = (tiles + reach - 1) / reach;
    const int64_t each = (tiles + chunks - 1) / chunks;
    f.chunk_rows = (int32_t)(each * rows);
    f.chunks = (int32_t)((tiles + each - 1) / each);
    return f;
}

struct Scratch { int64_t chunks, shares, bc; };          // floats of each, whole vectors but for the last
Scratch scratch_of(const SelScanParams &p, const Form &f, bool grad)
{
    Scratch s{};
    s.chunks = f.chunks > 1 ? (2 * f.chunks * p.B * p.D * p.N + 3) / 4 * 4 : 0;
    if (grad) {
        s.shares = f.chunks * p.B * share_floats(p);
        s.bc = f.slabs * p.B * p.T * 2 * p.N;
    }
    return s;
}
template <typename E, int R, bool KEEP, bool GATED>
void go(bool grad, const SelScanParams &p, const Form &f, float *shares, float *bc, hipStream_t s)
{
    const dim3 grid((unsigned)(p.B * f.slabs * f.chunks)), ahead((unsigned)(p.B * f.slabs * (f.chunks - 1))), wg(256);
    if (grad) {
        if (f.chunks > 1) hipLaunchKernelGGL((selective_scan_grad_kernel<E, R, KEEP, GATED, true>), ahead, wg, 0, s, p, f.slabs, f.chunks, f.chunk_rows, shares, bc);
        hipLaunchKernelGGL((selective_scan_grad_kernel<E, R, KEEP, GATED, false>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_rows, shares, bc);
    } else {
        if (f.chunks > 1) hipLaunchKernelGGL((selective_scan_kernel<E, R, KEEP, false, true>), ahead, wg, 0, s, p, f.slabs, f.chunks, f.chunk_rows);
        hipLaunchKernelGGL((selective_scan_kernel<E, R, KEEP, GATED, false>), grid, wg, 0, s, p, f.slabs, f.chunks, f.chunk_rows);
    }
}

template <typename E, int R>
hipError_t go(bool grad, const SelScanParams &p, const Form &f, hipStream_t s)
{
    const Scratch sc = scratch_of(p, f, grad);
    float *const shares = p.part ? p.part + sc.chunks : nullptr, *const bc = shares ? shares + sc.shares : nullptr;
    if (p.keep) p.z ? go<E, R, true, true>(grad, p, f, shares, bc, s) : go<E, R, true, false>(grad, p, f, shares, bc, s);
    else p.z ? go<E, R, false, true>(grad, p, f, shares, bc, s) : go<E, R, false, false>(grad, p, f, shares, bc, s);
    hipError_t er = hipGetLastError();
    if (er != hipSuccess || !grad) return er;
    SumShares q{};
    q.part = shares; q.P = f.chunks * p.B; q.stride = share_floats(p); q.dst_dtype = DT_F32;
    q.J = p.D * p.N + p.D; q.J1 = p.D * p.N; q.dst = p.da; q.dst2 = p.dskip;
    er = launch_sum_shares(q, s);
    if (er != hipSuccess) return er;
    q.part = bc; q.P = f.slabs; q.J = q.J1 = q.stride = p.B * p.T * 2 * p.N; q.dst = p.dbc; q.dst_dtype = p.dtype;
    return launch_sum_shares(q, s);
}

template <typename E> hipError_t go(bool grad, const SelScanParams &p, const Form &f, hipStream_t s)
{
    switch (f.R) {
    case 1: return go<E, 1>(grad, p, f, s);
    case 2: return go<E, 2>(grad, p, f, s);
    case 4: return go<E, 4>(grad, p, f, s);
    case 8: return go<E, 8>(grad, p, f, s);
    default: return go<E, 16>(grad, p, f, s);
    }
}

template <typename E, int R> void go_step(const SelScanParams &p, hipStream_t s)
{
    const int32_t slabs = (int32_t)((p.D + CHANNELS - 1) / CHANNELS);
    hipLaunchKernelGGL((selective_scan_step_kernel<E, R>), dim3((unsigned)(p.B * slabs)), dim3(256), 0, s, p, slabs);
}
template <typename E> hipError_t go_step(const SelScanParams &p, int R, hipStream_t s)
{
    switch (R) {
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
    const Form f = form_of(p, grad);
    // the sums over channels are a launch of a thousand threads a 64 columns
    return launch_has(p.B * f.slabs * f.chunks, 256) && (!grad || (p.B * p.T * 2 * p.N + 63) / 64 <= 0x3fffff);
}

int64_t sel_scan_state_rows(const SelScanParams &p) { return rows_of(form_of(p, true).R); }

int64_t sel_scan_part_floats(const SelScanParams &p, bool grad)
{
    const Scratch s = scratch_of(p, form_of(p, grad), grad);
    return s.chunks + s.shares + s.bc;
}

hipError_t launch_sel_scan(const SelScanParams &p, hipStream_t s)
{
    const Form f = form_of(p, false);
    if (!sel_scan_fits(p, false) || (f.chunks > 1 && !p.part) || p.gated != (p.z != nullptr) || p.keeps != (p.keep != nullptr)) return hipErrorInvalidValue;
    if (p.T == 1 && !p.states) {
        if (!p.y || !p.hT) return hipErrorInvalidValue;
        return p.dtype == DT_BF16 ? go_step<uint16_t>(p, f.R, s) : go_step<float>(p, f.R, s);
    }
    return p.dtype == DT_BF16 ? go<uint16_t>(false, p, f, s) : go<float>(false, p, f, s);
}

hipError_t launch_sel_scan_grad(const SelScanParams &p, hipStream_t s)
{
    if (!sel_scan_fits(p, true) || !p.part || !p.states || p.gated != (p.z != nullptr) || p.keeps != (p.keep != nullptr)) return hipErrorInvalidValue;
    const Form f = form_of(p, true);
    return p.dtype == DT_BF16 ? go<uint16_t>(true, p, f, s) : go<float>(true, p, f, s);
}

}  // namespace rl

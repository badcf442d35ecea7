// Short causal convolution over the rows of a sequence, every channel by itself:
//
//   u_t = b + sum_k w_k x_(t-K+1+k),   y_t = u_t or u_t sigmoid(u_t)
//
// over the sequence's tokens (rows whose keep is not 0), with the old state's K - 1 tokens before the first and nothing before a document's
// first token (keep 2).  Its gradient: g_t = dy_t act'(u_t), dx_t = sum_k w_k g_(t+K-1-k), dw_k = sum_t g_t x_(t-K+1+k), db = sum_t g_t.
//
// A wave owns 64 vectors of channels (16 bytes each, one element where rows do not start on 16 bytes) and a run of rows, which it walks with
// the last K - 1 tokens in registers; those before its run it finds by itself.  keep is the same for all lanes: a run's flags are two
// masks.  Of the gradient the wave also walks on behind its run, until its own tokens have all they get from later ones; its share of
// dw and db goes to memory, and a second launch adds the shares up, in a fixed order.
//
// Bound by the bytes that few waves have under way: two a SIMD are launched, and none follow those that have ended.  8 x 4096 x 2048 bf16, K 4, with the gate: forward 54 us
// (268 MB, 5.0 TB/s; 1.37 waves a SIMD are there on average, vector instructions take 35 % of its time), gradient 98 (403 MB, 4.1 TB/s; 0.88 waves, 56 %) and 5 of the
// shares; 1 x 16384 x 4096 in documents of some 400 tokens 63 to 68 (268 MB; 1.17 waves, 33 %).  One token of 64 sequences: 3.9 us, a launch's own time.
#include <type_traits>

#include "igemm_lds.h"

namespace rl {

namespace {

constexpr int RUN = 64;                       // rows of a run at most: a mask's bits
constexpr int AHEAD = 8;                      // rows asked for before the first of them is worked off; runs are of a multiple

template <typename E, int VEC> struct Row;
template <> struct Row<float, 4> { typedef u32x4 raw; };
template <> struct Row<uint16_t, 8> { typedef u32x4 raw; };
template <> struct Row<uint16_t, 4> { typedef u32x2 raw; };      // of more taps, whose window and sums take twice the registers
template <> struct Row<float, 1> { typedef uint32_t raw; };
template <> struct Row<uint16_t, 1> { typedef uint16_t raw; };

template <typename E, int VEC> __device__ __forceinline__ void unpack(const typename Row<E, VEC>::raw &r, float (&v)[VEC])
{
    if constexpr (VEC == 1 && sizeof(E) == 4) v[0] = __uint_as_float(r);
    else if constexpr (VEC == 1) v[0] = bf16_bits_to_f32(r);
    else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if constexpr (sizeof(E) == 4) v[j] = __uint_as_float(r[j]);
            else v[j] = __uint_as_float(j & 1 ? r[j >> 1] & 0xffff0000u : r[j >> 1] << 16);
        }
    }
}
template <typename E, int VEC> __device__ __forceinline__ typename Row<E, VEC>::raw pack(const float (&v)[VEC])
{
    typename Row<E, VEC>::raw r;
    if constexpr (VEC == 1 && sizeof(E) == 4) r = __float_as_uint(v[0]);
    else if constexpr (VEC == 1) r = (uint16_t)pack_bf16x2(v[0], v[0]);
    else {
#pragma unroll
        for (int j = 0; j < (int)(VEC * sizeof(E) / 4); ++j) {
            if constexpr (sizeof(E) == 4) r[j] = __float_as_uint(v[j]);
            else r[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
        }
    }
    return r;
}

// KT taps at most: K of them where KT < 8, else the last K (o = KT - K); slot j of KT - 1 holds the token KT - 1 - j before the present one
template <int KT> struct Taps {
    int o;
    __device__ __forceinline__ Taps(int K) : o(KT < 8 ? 0 : KT - K) {}
    __device__ __forceinline__ bool has(int j) const { return KT < 8 || j >= o; }
};

template <typename E, int VEC, int KT>
struct Walk {
    typedef typename Row<E, VEC>::raw raw_t;
    const CausalConvParams &p;
    Taps<KT> taps;
    int64_t b, d;
    int32_t run;
    bool live;
    float w[KT][VEC], bias[VEC];
    float win[KT - 1][VEC];

    __device__ __forceinline__ Walk(const CausalConvParams &p_, int32_t slabs, int32_t runs) : p(p_), taps((int)p_.K)
    {
        const uint32_t rest = blockIdx.x / (uint32_t)slabs;
        d = (int64_t)((blockIdx.x - rest * slabs) * 64 + threadIdx.x) * VEC;
        b = rest / (uint32_t)runs;
        run = (int32_t)(rest - (uint32_t)b * runs);
        live = d < p.D;
        if (!live) d = 0;                     // some other lane's channels, of which nothing is stored
        if constexpr (VEC > 1 && KT < 8) {
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                const f32x4 t = *(const f32x4 *)(p.b + d + j);
#pragma unroll
                for (int c = 0; c < 4; ++c) bias[j + c] = t[c];
            }
            // the channels' taps lie one behind the other, from a multiple of 16 bytes on
            if (p.w_dtype == DT_F32) {
#pragma unroll
                for (int i = 0; i < VEC * KT; i += 4) {
                    const f32x4 t = *(const f32x4 *)((const float *)p.w + d * KT + i);
#pragma unroll
                    for (int c = 0; c < 4; ++c) w[(i + c) % KT][(i + c) / KT] = t[c];
                }
            } else {
#pragma unroll
                for (int i = 0; i < VEC * KT; i += 8) {
                    const u32x4 t = *(const u32x4 *)((const uint16_t *)p.w + d * KT + i);
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (i + c < VEC * KT) w[(i + c) % KT][(i + c) / KT] = __uint_as_float(c & 1 ? t[c >> 1] & 0xffff0000u : t[c >> 1] << 16);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) bias[j] = p.b[d + j];
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[k][j] = taps.has(k) ? load_as_f32(p.w, p.w_dtype, (d + j) * p.K + k - taps.o) : 0.0f;
        }
    }
    __device__ __forceinline__ raw_t row(const void *x, int64_t t) const { return *(const raw_t *)((const E *)x + (b * p.T + t) * p.D + d); }
    __device__ __forceinline__ raw_t state(const void *s, int j) const { return *(const raw_t *)((const E *)s + (b * (p.K - 1) + j - taps.o) * p.D + d); }
    __device__ __forceinline__ void put(void *x, int64_t t, const float (&v)[VEC]) const
    {
        raw_t *const to = (raw_t *)((E *)x + (b * p.T + t) * p.D + d);
        if (!live) return;
        if constexpr (VEC > 1) __builtin_nontemporal_store(pack<E, VEC>(v), to);
        else *to = pack<E, VEC>(v);
    }
    __device__ __forceinline__ void put_state(void *s, int j, const float (&v)[VEC]) const
    {
        if (live) *(raw_t *)((E *)s + (b * (p.K - 1) + j - taps.o) * p.D + d) = pack<E, VEC>(v);
    }
    // flags of the up to 64 rows from t on: bit i set where row t + i is a token, a document's first
    __device__ __forceinline__ void flags(int64_t t, int64_t rows, uint64_t &tok, uint64_t &first) const
    {
        const int i = threadIdx.x & 63;
        const int k = i < rows ? p.keep[b * p.T + t + i] : 0;
        tok = __ballot(k != 0);
        first = __ballot(k == 2);
    }
    // whether there is a token among the 256 rows from t on
    __device__ __forceinline__ bool any(int64_t t) const
    {
        int some = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) some |= p.keep[b * p.T + t + 64 * q + (threadIdx.x & 63)];
        return __ballot(some != 0) != 0;
    }
    // the tokens before row t0
    template <bool KEEP> __device__ __forceinline__ void before(int64_t t0)
    {
#pragma unroll
        for (int j = 0; j < KT - 1; ++j)
#pragma unroll
            for (int v = 0; v < VEC; ++v) win[j][v] = 0.0f;
        if constexpr (!KEEP) {
#pragma unroll
            for (int j = 0; j < KT - 1; ++j) {
                if (!taps.has(j)) continue;
                const int64_t t = t0 - (KT - 1) + j;
                unpack<E, VEC>(t >= 0 ? row(p.x, t) : state(p.s0, (int)(t0 + j)), win[j]);
            }
        } else {
            int have = 0;                     // tokens found, the newest first
            const int want = (int)p.K - 1;
            bool open = true;                 // no document's first token among them
            int64_t end = t0;
            while (end >= 256 && !any(end - 256)) end -= 256;        // long padding
            for (; end > 0 && have < want && open; end -= 64) {
                const int64_t t = end > 64 ? end - 64 : 0;
                uint64_t tok, first;
                flags(t, end - t, tok, first);
                while (tok && have < want && open) {
                    const int i = 63 - __builtin_clzll(tok);
                    tok &= ~(1ull << i);
                    set(KT - 2 - have, row(p.x, t + i));
                    ++have;
                    open = !(first >> i & 1);
                }
            }
            if (open) {
#pragma unroll
                for (int j = 0; j < KT - 1; ++j)      // slot j takes the state's token have slots on
                    if (taps.has(j) && j + have < KT - 1) unpack<E, VEC>(state(p.s0, j + have), win[j]);
            }
        }
    }
    __device__ __forceinline__ void set(int slot, const raw_t &r)
    {
        // values chosen, not places: places chosen would put the window into memory
        float x[VEC];
        unpack<E, VEC>(r, x);
#pragma unroll
        for (int j = 0; j < KT - 1; ++j)
#pragma unroll
            for (int v = 0; v < VEC; ++v) win[j][v] = j == slot ? x[v] : win[j][v];
    }
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int j = 0; j < KT - 1; ++j)
#pragma unroll
            for (int v = 0; v < VEC; ++v) win[j][v] = 0.0f;
    }
    __device__ __forceinline__ void sum(const float (&x)[VEC], float (&u)[VEC]) const
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) u[v] = bias[v];
#pragma unroll
        for (int j = 0; j < KT - 1; ++j) {
            if (!taps.has(j)) continue;
#pragma unroll
            for (int v = 0; v < VEC; ++v) u[v] = __builtin_fmaf(w[j][v], win[j][v], u[v]);
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) u[v] = __builtin_fmaf(w[KT - 1][v], x[v], u[v]);
    }
    __device__ __forceinline__ void shift(const float (&x)[VEC])
    {
#pragma unroll
        for (int j = 0; j < KT - 1; ++j)
#pragma unroll
            for (int v = 0; v < VEC; ++v) win[j][v] = !taps.has(j) ? 0.0f : j + 1 < KT - 1 ? win[j + 1 < KT - 1 ? j + 1 : j][v] : x[v];
    }
};

// u sigmoid(u); for u below -87 at 0 times the rest: -0
__device__ __forceinline__ float silu(float u) { return u * sigmoidf_(u); }
// its derivative
__device__ __forceinline__ float silu_slope(float u)
{
    const float s = sigmoidf_(u);
    return __builtin_fmaf(u * s, sigmoidf_(-u), s);
}

}  // namespace

template <typename E, int VEC, int KT, bool KEEP>
__global__ __launch_bounds__(64) void causal_conv_kernel(const CausalConvParams p, int32_t slabs, int32_t runs, int32_t rows)
{
    typedef Walk<E, VEC, KT> W;
    typedef typename W::raw_t raw_t;
    W k(p, slabs, runs);
    const int64_t t0 = (int64_t)k.run * rows, left = p.T - t0;
    const int n = (int)(left < rows ? left : rows);
    uint64_t tok = ~0ull, first = 0;
    if (KEEP) k.flags(t0, n, tok, first);
    const bool last = k.run + 1 == runs;
    if (!KEEP || tok || last) k.template before<KEEP>(t0);
    auto walk = [&](auto plain) __attribute__((always_inline)) {                 // plain: the rows are all there, and tokens of one document
        raw_t r[2][AHEAD];
        auto ask = [&](raw_t (&q)[AHEAD], int i) __attribute__((always_inline)) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) q[a] = k.row(p.x, t0 + (i + a < n ? i + a : n - 1));
        };
        auto rows_of = [&](const raw_t (&q)[AHEAD], int i) __attribute__((always_inline)) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                float x[VEC], u[VEC];
                if (!plain && i + a >= n) continue;
                if (!plain && !(tok >> (i + a) & 1)) {
#pragma unroll
                    for (int v = 0; v < VEC; ++v) u[v] = 0.0f;
                    k.put(p.y, t0 + i + a, u);
                    continue;
                }
                if (!plain && (first >> (i + a) & 1)) k.forget();
                unpack<E, VEC>(q[a], x);
                k.sum(x, u);
                if (p.silu) {
#pragma unroll
                    for (int v = 0; v < VEC; ++v) u[v] = silu(u[v]);
                }
                k.put(p.y, t0 + i + a, u);
                k.shift(x);
            }
        };
        ask(r[0], 0);
        for (int i = 0; i < n; i += 2 * AHEAD) {
            if (i + AHEAD < n) ask(r[1], i + AHEAD);
            rows_of(r[0], i);
            if (i + 2 * AHEAD < n) ask(r[0], i + 2 * AHEAD);
            if (i + AHEAD < n) rows_of(r[1], i + AHEAD);
        }
    };
    const uint64_t all = n == 64 ? ~0ull : (1ull << n) - 1;
    if (n == rows && (tok & all) == all && first == 0) walk(std::true_type{});
    else walk(std::false_type{});
    if (last) {
#pragma unroll
        for (int j = 0; j < KT - 1; ++j)
            if (k.taps.has(j)) k.put_state(p.sT, j, k.win[j]);
    }
}

template <typename E, int VEC, int KT, bool KEEP>
__global__ __launch_bounds__(64) void causal_conv_grad_kernel(const CausalConvParams p, int32_t slabs, int32_t runs, int32_t rows)
{
    typedef Walk<E, VEC, KT> W;
    typedef typename W::raw_t raw_t;
    W k(p, slabs, runs);
    const int64_t t0 = (int64_t)k.run * rows, left = p.T - t0;
    const int n = (int)(left < rows ? left : rows);
    uint64_t tok = ~0ull, first = 0;
    if (KEEP) k.flags(t0, n, tok, first);
    float dw[KT][VEC], db[VEC], pend[KT - 1][VEC];
    int64_t pos[KT - 1];                          // the row a slot's derivative goes to; NOT_MINE, or of the state's token j STATE - j
    constexpr int64_t NOT_MINE = -1, STATE = -2;
#pragma unroll
    for (int v = 0; v < VEC; ++v) db[v] = 0.0f;
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
        for (int v = 0; v < VEC; ++v) dw[j][v] = 0.0f;
    int owed = 0;                                 // slots that are mine
#pragma unroll
    for (int j = 0; j < KT - 1; ++j) {
        const bool mine = k.run == 0 && k.taps.has(j);
        pos[j] = mine ? STATE - j : NOT_MINE;
        owed += mine;
#pragma unroll
        for (int v = 0; v < VEC; ++v) pend[j][v] = 0.0f;
    }
    auto flush = [&](int j) __attribute__((always_inline)) {
        if (pos[j] >= 0) k.put(p.dx, pos[j], pend[j]);
        else if (pos[j] <= STATE) k.put_state(p.ds0, (int)(STATE - pos[j]), pend[j]);
        owed -= pos[j] != NOT_MINE;
    };
    auto forget = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < KT - 1; ++j) {
            flush(j);
            pos[j] = NOT_MINE;
#pragma unroll
            for (int v = 0; v < VEC; ++v) pend[j][v] = 0.0f;
        }
        k.forget();
    };
    // a token at row t, one of the run's own or behind it.  plain: all of the run before it are tokens, so that slots' rows are known
    auto token = [&](int64_t t, const raw_t &rx, const raw_t &rdy, bool mine, auto plain) __attribute__((always_inline)) {
        float x[VEC], g[VEC], u[VEC];
        unpack<E, VEC>(rx, x);
        unpack<E, VEC>(rdy, g);
        if (p.silu) {
            k.sum(x, u);
#pragma unroll
            for (int v = 0; v < VEC; ++v) g[v] *= silu_slope(u[v]);
        }
        if (mine) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                db[v] += g[v];
                dw[KT - 1][v] = __builtin_fmaf(g[v], x[v], dw[KT - 1][v]);
#pragma unroll
                for (int j = 0; j < KT - 1; ++j)
                    if (k.taps.has(j)) dw[j][v] = __builtin_fmaf(g[v], k.win[j][v], dw[j][v]);
            }
        }
#pragma unroll
        for (int j = 0; j < KT - 1; ++j) {
            if (!k.taps.has(j)) continue;
#pragma unroll
            for (int v = 0; v < VEC; ++v) pend[j][v] = __builtin_fmaf(k.w[j][v], g[v], pend[j][v]);
        }
        if (plain) {
            const int64_t i = t - t0;
            if (i >= KT - 1) k.put(p.dx, t - (KT - 1), pend[0]);
            else if (k.run == 0) k.put_state(p.ds0, (int)i, pend[0]);
        } else {
#pragma unroll
            for (int j = 0; j < KT - 1; ++j)
                if (j == k.taps.o) flush(j);
        }
#pragma unroll
        for (int j = 0; j < KT - 1; ++j) {
            const bool end = j + 1 == KT - 1;
            if (!plain) pos[j] = !k.taps.has(j) ? NOT_MINE : end ? (mine ? t : NOT_MINE) : pos[end ? j : j + 1];
#pragma unroll
            for (int v = 0; v < VEC; ++v) pend[j][v] = !k.taps.has(j) ? 0.0f : end ? k.w[KT - 1][v] * g[v] : pend[end ? j : j + 1][v];
        }
        if (!plain) owed += mine;
        k.shift(x);
    };
    if (!KEEP || tok || owed) k.template before<KEEP>(t0);
    constexpr int SOME = AHEAD / 2;               // of two tensors
    auto walk = [&](auto plain) __attribute__((always_inline)) {
        raw_t r[2][SOME], q[2][SOME];
        auto ask = [&](int s, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int a = 0; a < SOME; ++a) {
                const int64_t t = t0 + (i + a < n ? i + a : n - 1);
                r[s][a] = k.row(p.x, t);
                q[s][a] = k.row(p.dy, t);
            }
        };
        auto rows_of = [&](auto half, int i) __attribute__((always_inline)) {
            constexpr int S = decltype(half)::value;
#pragma unroll
            for (int a = 0; a < SOME; ++a) {
                if (!plain && i + a >= n) continue;
                if (!plain && !(tok >> (i + a) & 1)) {
                    float zero[VEC];
#pragma unroll
                    for (int v = 0; v < VEC; ++v) zero[v] = 0.0f;
                    k.put(p.dx, t0 + i + a, zero);
                    continue;
                }
                if (!plain && (first >> (i + a) & 1)) forget();
                token(t0 + i + a, r[S][a], q[S][a], true, plain);
            }
        };
        ask(0, 0);
        for (int i = 0; i < n; i += 2 * SOME) {
            if (i + SOME < n) ask(1, i + SOME);
            rows_of(std::integral_constant<int, 0>{}, i);
            if (i + 2 * SOME < n) ask(0, i + 2 * SOME);
            if (i + SOME < n) rows_of(std::integral_constant<int, 1>{}, i + SOME);
        }
    };
    const uint64_t all = n == 64 ? ~0ull : (1ull << n) - 1;
    if (KT < 8 && n == rows && (tok & all) == all && first == 0) {
        walk(std::true_type{});
#pragma unroll
        for (int j = 0; j < KT - 1; ++j) pos[j] = t0 + n - (KT - 1) + j;
        owed = KT - 1;
    } else {
        walk(std::false_type{});
    }
    // what later tokens give to mine
    int64_t t = t0 + n;
    if (KEEP) {
        while (owed && t + 256 <= p.T && !k.any(t)) t += 256;
    }
    for (; owed && t < p.T; t += 64) {
        const int64_t m = p.T - t < 64 ? p.T - t : 64;
        uint64_t more = m == 64 ? ~0ull : (1ull << m) - 1, starts = 0;
        if (KEEP) k.flags(t, m, more, starts);
        while (more && owed) {
            const int i = __builtin_ctzll(more);
            more &= more - 1;
            if (KEEP && (starts >> i & 1)) { forget(); break; }
            token(t + i, k.row(p.x, t + i), k.row(p.dy, t + i), false, std::false_type{});
        }
    }
    if (owed) {                                   // the sequence's end: the new state's derivative is theirs
#pragma unroll
        for (int j = 0; j < KT - 1; ++j) {
            if (!k.taps.has(j) || pos[j] == NOT_MINE) continue;
            float ds[VEC];
            unpack<E, VEC>(k.state(p.dsT, j), ds);
#pragma unroll
            for (int v = 0; v < VEC; ++v) pend[j][v] += ds[v];
            flush(j);
        }
    }
    if (k.live) {
        float *part = p.part + (k.b * runs + k.run) * (p.K + 1) * p.D + k.d;
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            if (!k.taps.has(j)) continue;
#pragma unroll
            for (int v = 0; v < VEC; ++v) part[(j - k.taps.o) * p.D + v] = dw[j][v];
        }
#pragma unroll
        for (int v = 0; v < VEC; ++v) part[p.K * p.D + v] = db[v];
    }
}

// ---------------------------------------------------------------------------
// sums of shares, sixteen of them under way at a time a column
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void sum_shares_kernel(const SumShares q)
{
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t j = (int64_t)blockIdx.x * 64 + lane;
    float v = 0.0f;
    if (j < q.J) {
#pragma unroll 8
        for (int64_t i = wave; i < q.P; i += 16) v += q.part[i * q.stride + j];
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && j < q.J) {
#pragma unroll
        for (int w = 1; w < 16; ++w) v += s[w][lane];
        // rows of `turn` columns become columns of `across` rows
        const int64_t at = q.turn ? (j % q.turn) * q.across + j / q.turn : j;
        if (j < q.J1) store_from_f32(q.dst, q.dst_dtype, at, v);
        else q.dst2[j - q.J1] = v;
    }
}

// many columns: VEC of them a thread, one share after the other
template <int VEC>
__global__ __launch_bounds__(256) void sum_columns_kernel(const SumShares q)
{
    const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * VEC;
    if (j >= q.J) return;
    if constexpr (VEC == 4) {
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (int64_t i = 0; i < q.P; ++i) v += *(const f32x4 *)(q.part + i * q.stride + j);
        if (q.dst_dtype == DT_BF16) *(u32x2 *)((uint16_t *)q.dst + j) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else *(f32x4 *)((float *)q.dst + j) = v;
    } else {
        float v = 0.0f;
#pragma unroll 8
        for (int64_t i = 0; i < q.P; ++i) v += q.part[i * q.stride + j];
        store_from_f32(q.dst, q.dst_dtype, j, v);
    }
}

hipError_t launch_sum_shares(const SumShares &q, hipStream_t s)
{
    if (q.J < 1 || q.P < 1 || (q.J + 63) / 64 > 0x3fffff) return hipErrorInvalidValue;
    // few shares of many columns: a thread of its own for every four (67 MB in 32 shares of 524288 columns 30 -> 12 us); where columns are few, sixteen waves share one's shares
    if (q.J >= (1 << 16) && q.P <= 256 && q.J1 == q.J && !q.turn) {
        if (q.J % 4 == 0 && q.stride % 4 == 0 && ((uintptr_t)q.part | (uintptr_t)q.dst) % 16 == 0)
            hipLaunchKernelGGL((sum_columns_kernel<4>), dim3((unsigned)((q.J / 4 + 255) / 256)), dim3(256), 0, s, q);
        else
            hipLaunchKernelGGL((sum_columns_kernel<1>), dim3((unsigned)((q.J + 255) / 256)), dim3(256), 0, s, q);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(sum_shares_kernel, dim3((unsigned)((q.J + 63) / 64)), dim3(1024), 0, s, q);
    return hipGetLastError();
}

namespace {

struct Form { int32_t slabs, runs, rows, vec; };

Form form_of(const CausalConvParams &p)
{
    Form f;
    const int whole = p.dtype == DT_BF16 && p.K <= 4 ? 8 : 4;
    f.vec = p.D % whole == 0 ? whole : 1;
    f.slabs = (int32_t)((p.D + 64 * f.vec - 1) / (64 * f.vec));
    // long runs read fewer tokens before them and leave fewer shares, short ones fill the CUs: eight waves of each
    f.rows = RUN;
    while (f.rows > 16 && p.B * f.slabs * ((p.T + f.rows - 1) / f.rows) < 2048) f.rows /= 2;
    f.runs = (int32_t)((p.T + f.rows - 1) / f.rows);
    return f;
}

template <typename E, int VEC, int KT>
void go(bool grad, const CausalConvParams &p, const Form &f, hipStream_t s)
{
    const dim3 grid((unsigned)(p.B * f.slabs * f.runs)), wg(64);
    if (grad) {
        if (p.keep) hipLaunchKernelGGL((causal_conv_grad_kernel<E, VEC, KT, true>), grid, wg, 0, s, p, f.slabs, f.runs, f.rows);
        else hipLaunchKernelGGL((causal_conv_grad_kernel<E, VEC, KT, false>), grid, wg, 0, s, p, f.slabs, f.runs, f.rows);
    } else {
        if (p.keep) hipLaunchKernelGGL((causal_conv_kernel<E, VEC, KT, true>), grid, wg, 0, s, p, f.slabs, f.runs, f.rows);
        else hipLaunchKernelGGL((causal_conv_kernel<E, VEC, KT, false>), grid, wg, 0, s, p, f.slabs, f.runs, f.rows);
    }
}

template <typename E, int VEC>
void go(bool grad, const CausalConvParams &p, const Form &f, hipStream_t s)
{
    if (p.K > 4) {
        go<E, (VEC < 4 ? VEC : 4), 8>(grad, p, f, s);
        return;
    }
    if (p.K == 2) go<E, VEC, 2>(grad, p, f, s);
    else if (p.K == 3) go<E, VEC, 3>(grad, p, f, s);
    else go<E, VEC, 4>(grad, p, f, s);
}

hipError_t go(bool grad, const CausalConvParams &p, const Form &f, hipStream_t s)
{
    if (p.dtype == DT_BF16) f.vec > 1 ? go<uint16_t, 8>(grad, p, f, s) : go<uint16_t, 1>(grad, p, f, s);
    else f.vec > 1 ? go<float, 4>(grad, p, f, s) : go<float, 1>(grad, p, f, s);
    return hipGetLastError();
}

}  // namespace

bool causal_conv_fits(const CausalConvParams &p)
{
    if (p.B < 1 || p.T < 1 || p.D < 1 || p.K < 2 || p.K > 8 || p.B > 0x7fffffff || p.T > 0x7fffffff || p.D > SCAN_MAX_D) return false;
    const Form f = form_of(p);
    return launch_has((int64_t)f.slabs * f.runs, 64) && launch_has(p.B * f.slabs * f.runs, 64);
}

int64_t causal_conv_part_floats(const CausalConvParams &p)
{
    return p.B * form_of(p).runs * (p.K + 1) * p.D;
}

hipError_t launch_causal_conv(const CausalConvParams &p, hipStream_t s)
{
    if (!causal_conv_fits(p)) return hipErrorInvalidValue;
    return go(false, p, form_of(p), s);
}

hipError_t launch_causal_conv_grad(const CausalConvParams &p, hipStream_t s)
{
    if (!causal_conv_fits(p) || !p.part) return hipErrorInvalidValue;
    const Form f = form_of(p);
    hipError_t er = go(true, p, f, s);
    if (er != hipSuccess) return er;
    SumShares q{};
    q.part = p.part; q.P = p.B * f.runs; q.stride = (p.K + 1) * p.D;
    q.J = (p.K + 1) * p.D; q.J1 = p.K * p.D; q.turn = p.D; q.across = p.K; q.dst = p.dw; q.dst_dtype = DT_F32; q.dst2 = p.db;
    return launch_sum_shares(q, s);
}

}  // namespace rl

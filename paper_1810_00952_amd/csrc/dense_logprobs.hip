// Token log probabilities over a large vocabulary, from the last layer's rows x[M, K] and the vocabulary's w[V, K], and their gradients, without
// the logits l = x w^T in memory:
//
//   lse = ln sum_v e^l,  lp = l[tok] - lse;   dl = dlp (1[v = tok] - p) + dlse p,  p = e^(l - lse);   dx = dl w,  dw = dl^T x
//
// Forward: a product's tile leaves a maximum and a sum of exponentials a row, and the token's logit where it is its column; a second launch joins
// them.  Gradient, for pieces of the vocabulary: the piece's logits once more, dl from them, rounded to x's type as a product's operand and stored
// as it lies and transposed; then dx += dl w and dw = dl^T x, all three products of rows that lie along the contraction.  x and w are
// transposed for the last two.
#include "igemm_lds.h"

namespace rl {

namespace {

struct NtParams {                             // c[m, n] = sum_k x[m, k] w[n, k]; rows ldx, ldw bytes apart, kbytes of them (multiples of 16) count
    const void *x, *w;
    int64_t M, N, ldx, ldw;
    int32_t kbytes;
    int32_t nblk_m, nblk_n, nk;               // tiles along x and w, 128-byte lines of a row
    int32_t split_lines;                      // lines of a slice of K (grid's y: slices)
};

template <typename E> struct Mfma;
template <> struct Mfma<uint16_t> {
    static __device__ __forceinline__ void go(f32x16 &c, const u32x4 &a, const u32x4 &b)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<float> {
    static __device__ __forceinline__ void go(f32x16 &c, const u32x4 &a, const u32x4 &b)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    }
};

// (m, s): s e^m stands for a sum of exponentials; m -inf: of none
struct Soft { float m, s; };
__device__ __forceinline__ Soft join(Soft a, Soft b)
{
    const float m = fmaxf(a.m, b.m);
    const float fa = a.m == m ? 1.0f : __expf(a.m - m), fb = b.m == m ? 1.0f : __expf(b.m - m);
    return {m, __builtin_fmaf(a.s, fa, b.s * fb)};
}

// ---- what becomes of a tile's sums.  A lane has row m of x and of w's rows n = n0 + 8 k + i, k, i < 4 (n0 counts the lane's half) --------------
struct StatsEpi {
    float2 *part; float *hit; const int32_t *tok; int64_t M, V;
    static constexpr bool STATS = true;
};
template <typename E> struct GradEpi {
    E *g, *gt; int64_t ldg, ldgt;             // elements
    const int32_t *tok; const float *lse, *dlp, *dlse;
    int64_t M, V, v0, Vp, Mp;                 // columns v0 .. of the vocabulary; Vp of them are written, Mp rows
    static constexpr bool STATS = false;
    struct Row { float lse, one, all; int32_t tok; };
    __device__ __forceinline__ Row row(int64_t m) const
    {
        Row r{0.0f, 0.0f, 0.0f, -1};
        if (m >= M) return r;
        r.tok = tok[m];
        const bool given = r.tok >= 0 && r.tok < V;
        r.lse = lse[m] == -INFINITY ? INFINITY : lse[m];      // of no logits: p is 0
        r.one = given ? dlp[m] : 0.0f;
        r.all = dlse[m] - r.one;
        return r;
    }
    __device__ __forceinline__ void put(int64_t m, int64_t n, const f32x4 &l, const Row &r) const
    {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t col = v0 + n + i;
            const float p = __expf(l[i] - r.lse);
            v[i] = (r.one == 0.0f && r.all == 0.0f) || col >= V ? 0.0f : __builtin_fmaf(r.all, p, col == r.tok ? r.one : 0.0f);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i >= Vp) continue;
            if (m < M) store(g, m * ldg + n + i, v[i]);
            if (m < Mp) store(gt, (n + i) * ldgt + m, v[i]);
        }
    }
    static __device__ __forceinline__ void store(E *p, int64_t i, float v)
    {
        if constexpr (sizeof(E) == 4) p[i] = v;
        else p[i] = (uint16_t)pack_bf16x2(v, v);
    }
};
// c (+ what was added up before) to y or, of a slice of K, to its share
struct OutEpi {
    void *y; const float *before; float *sum;  // sum: f32, in place of y
    int64_t M, N; int32_t y_dtype;
    static constexpr bool STATS = false;
    struct Row {};
    __device__ __forceinline__ Row row(int64_t) const { return {}; }
    __device__ __forceinline__ void put(int64_t m, int64_t n, const f32x4 &c, const Row &) const
    {
        if (m >= M) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i >= N) continue;
            const int64_t at = m * N + n + i;
            const float v = before ? c[i] + before[at] : c[i];
            if (sum) sum[at + (int64_t)blockIdx.y * M * N] = v;
            else store_from_f32(y, y_dtype, at, v);
        }
    }
};

}  // namespace

// ---------------------------------------------------------------------------
// WM x WN waves, each TM x TN groups of 32 rows of x and of w
// ---------------------------------------------------------------------------
template <typename E, int WM, int WN, int TM, int TN, typename Epi>
__global__ __launch_bounds__(64 * WM * WN) void nt_tile_kernel(const NtParams p, const Epi epi)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, W = WM * WN, X_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    constexpr int LPT = (BM + BN) / 8 / W, XL = BM / 8 / W;        // direct loads per wave and tile, those of x first
    static_assert((BM / 8) % W == 0 && (BN / 8) % W == 0 && LPT % 2 == 0, "a tile's loads in whole halves of every wave's");
    __shared__ __attribute__((aligned(1024))) unsigned char st0[STAGE];
    __shared__ __attribute__((aligned(1024))) unsigned char st1[STAGE];

    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // each XCD a contiguous run of tiles; inside a run, column tiles in groups of eight with the row tiles fastest
    int32_t bm, bn;
    {
        constexpr int GN = 8;
        const int32_t bid = xcd_run(blockIdx.x, p.nblk_m * p.nblk_n), grp = bid / (GN * p.nblk_m), within = bid - grp * GN * p.nblk_m;
        const int32_t gw = min(GN, p.nblk_n - grp * GN);
        bm = within / gw; bn = grp * GN + (within - bm * gw);
    }
    const int64_t m0 = (int64_t)bm * BM, n0 = (int64_t)bn * BN;
    // from the tile's first rows on: offsets stay small whatever the matrices' sizes
    const int64_t xroom = min((p.M - m0) * p.ldx, (int64_t)0x7fffffff), wroom = min((p.N - n0) * p.ldw, (int64_t)0x7fffffff);
    const rsrc_t rx = make_rsrc((const char *)p.x + m0 * p.ldx, (uint32_t)xroom), rw = make_rsrc((const char *)p.w + n0 * p.ldw, (uint32_t)wroom);

    // lane l of a load fills row l >> 3, position l & 7 of eight rows of 128 bytes; chunks of 16 swizzled by the row
    uint32_t voff[LPT];
    int32_t room[LPT];                            // bytes of the row from the lane's chunk on
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
        const bool x = i < XL;
        const int row = x ? (wave * XL + i) * 8 + (lane >> 3) : (wave * (LPT - XL) + i - XL) * 8 + (lane >> 3);
        const int chunk = (lane & 7) ^ ((row >> 1) & 7);
        const bool in = x ? m0 + row < p.M : n0 + row < p.N;
        voff[i] = in ? (uint32_t)row * (uint32_t)(x ? p.ldx : p.ldw) + chunk * 16 : OOB;
        room[i] = in ? p.kbytes - chunk * 16 : 0;
    }
    int32_t f_kt = blockIdx.y * p.split_lines;
    const int32_t end = min(f_kt + p.split_lines, p.nk), lines = end - f_kt;
    int32_t f_at = 0;
    bool f_live = true;
    auto begin = [&]() { f_live = f_kt < end; f_at = f_live ? f_kt * 128 : 0; ++f_kt; };
    auto dma = [&](unsigned char *st, int d) {
        unsigned char *to = d < XL ? st + (wave * XL + d) * 1024 : st + X_BYTES + (wave * (LPT - XL) + d - XL) * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d < XL ? rx : rw, RL_LDS_PTR(to), 16, f_live && f_at < room[d] ? voff[d] + f_at : OOB, 0, 0, 0);
    };

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;
    const int frow = lane & 31, fhalf = lane >> 5;
    int f_off[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) f_off[ks] = frow * 128 + (((2 * ks + fhalf) ^ ((frow >> 1) & 7)) << 4);
    u32x4 fw[2][TN], fx[2][TM];
    auto fragments = [&](const unsigned char *st, int ks) {
#pragma unroll
        for (int j = 0; j < TN; ++j) fw[ks & 1][j] = *(const u32x4 *)(st + X_BYTES + (wn * TN + j) * 4096 + f_off[ks]);
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[ks & 1][i] = *(const u32x4 *)(st + (wm * TM + i) * 4096 + f_off[ks]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // a k-step's MFMAs; req 0, 1: the first, second half of a tile's direct loads between them, 2: none
    auto multiply = [&](int ks, unsigned char *to, int req) {
        constexpr int HALF = LPT / 2, N = TM * TN;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                Mfma<E>::go(acc[i][j], fw[ks & 1][j], fx[ks & 1][i]);
                if (req < 2) {
                    const int n = i * TN + j;
#pragma unroll
                    for (int d = n * HALF / N; d < (n + 1) * HALF / N; ++d) dma(to, req * HALF + d);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    // tile t in cur, the first half of tile t + 1's loads under way into nxt
    auto body = [&](unsigned char *cur, unsigned char *nxt) {
        fragments(cur, 1);
        multiply(0, nxt, 1);
        fragments(cur, 2);
        multiply(1, cur, 2);
        fragments(cur, 3);
        multiply(2, cur, 2);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        begin();
        fragments(nxt, 0);
        multiply(3, cur, 0);
    };
    begin();
#pragma unroll
    for (int d = 0; d < LPT; ++d) dma(st0, d);
    begin();
#pragma unroll
    for (int d = 0; d < LPT / 2; ++d) dma(st1, d);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LPT / 2) : "memory");
    fragments(st0, 0);
    int32_t kt = 0;
#pragma unroll 1
    for (; kt + 2 <= lines; kt += 2) {
        body(st0, st1);
        body(st1, st0);
    }
    if (kt < lines) body(st0, st1);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");      // the trailing requests; from here the stages are free

    if constexpr (Epi::STATS) {
        Soft *const seen = (Soft *)st0;                             // [WN][BM]
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + (wm * TM + i) * 32 + frow;
            const int32_t tok = m < epi.M ? epi.tok[m] : -1;
            Soft s{-INFINITY, 0.0f};
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t nj = n0 + (wn * TN + j) * 32 + 4 * fhalf;
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int64_t n = nj + 8 * (q >> 2) + (q & 3);
                    const float l = n < epi.V ? acc[i][j][q] : -INFINITY;
                    acc[i][j][q] = l;
                    if (n == tok && n < epi.V) epi.hit[m] = l;
                    s.m = fmaxf(s.m, l);
                }
            }
            // of NaN a maximum is the other number: the sum has it
            const float top = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) s.s += __expf(acc[i][j][q] - top);
            Soft o{__shfl_xor(s.m, 32), __shfl_xor(s.s, 32)};
            s = join(s, o);
            if (fhalf == 0) seen[wn * BM + (wm * TM + i) * 32 + frow] = s;
        }
        __syncthreads();
        for (int r = t; r < BM; r += 64 * W) {
            if (m0 + r >= epi.M) break;
            Soft s = seen[r];
#pragma unroll
            for (int w = 1; w < WN; ++w) s = join(s, seen[w * BM + r]);
            epi.part[(int64_t)bn * epi.M + m0 + r] = float2{s.m, s.s};
        }
    } else {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + (wm * TM + i) * 32 + frow;
            const auto row = epi.row(m);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    epi.put(m, n0 + (wn * TN + j) * 32 + 8 * k + 4 * fhalf, f32x4{acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]}, row);
        }
    }
#endif
}

// ---------------------------------------------------------------------------
// rows' sums of all tiles; eight threads a row
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void dense_logprobs_join_kernel(const float2 *part, const float *hit, const int32_t *tok, float *lp, float *lse, int64_t M, int64_t V, int32_t tiles)
{
    __shared__ Soft seen[8][32];
    const int r = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int64_t m = (int64_t)blockIdx.x * 32 + r;
    Soft s{-INFINITY, 0.0f};
    if (m < M)
        for (int32_t t = share; t < tiles; t += 8) {
            const float2 v = part[(int64_t)t * M + m];
            s = join(s, Soft{v.x, v.y});
        }
    seen[share][r] = s;
    __syncthreads();
    if (share == 0 && m < M) {
#pragma unroll
        for (int k = 1; k < 8; ++k) s = join(s, seen[k][r]);
        const float all = s.m == INFINITY ? __uint_as_float(0x7fc00000u) : s.m + __logf(s.s);
        const int32_t at = tok[m];
        lse[m] = all;
        lp[m] = at < 0 || at >= V ? 0.0f : all == -INFINITY ? -INFINITY : hit[m] - all;
    }
}

// ---------------------------------------------------------------------------
// src[R][C] (rows ld elements apart) -> dst[C][Rp], zeros behind R; rows without a derivative are zeros
// ---------------------------------------------------------------------------
template <typename E>
__global__ __launch_bounds__(256) void turn_rows_kernel(const E *src, E *dst, int64_t Rr, int64_t C, int64_t ld, int64_t Rp, const int32_t *tok, const float *dlp, const float *dlse, int64_t V)
{
    __shared__ E s[64][65];
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;
    const int c = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int r = w; r < 64; r += 4) {
        E v = 0;
        if (r0 + r < Rr && c0 + c < C) {
            bool part = true;
            if (tok) {
                const int32_t k = tok[r0 + r];
                part = dlse[r0 + r] != 0.0f || (k >= 0 && k < V && dlp[r0 + r] != 0.0f);
            }
            if (part) v = src[(r0 + r) * ld + c0 + c];
        }
        s[r][c] = v;
    }
    __syncthreads();
    for (int k = w; k < 64; k += 4)
        if (c0 + k < C && r0 + c < Rp) dst[(c0 + k) * Rp + r0 + c] = s[c][k];
}

namespace {

constexpr int64_t LINE = 128, PIECE_MAX = 1 << 20;      // a piece's columns: a row of dl is reached by 31-bit offsets from its tile's first
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
size_t esize(const DenseLogprobsParams &p) { return p.dtype == DT_BF16 ? 2 : 4; }

template <typename E, typename Epi>
void go_nt(NtParams q, const Epi &epi, int32_t splits, hipStream_t s)
{
    q.nblk_m = (int32_t)((q.M + 127) / 128);
    q.nblk_n = (int32_t)((q.N + 127) / 128);
    q.nk = (int32_t)((q.kbytes + LINE - 1) / LINE);
    q.split_lines = (q.nk + splits - 1) / splits;
    hipLaunchKernelGGL((nt_tile_kernel<E, 2, 2, 2, 2, Epi>), dim3((unsigned)((int64_t)q.nblk_m * q.nblk_n), (unsigned)splits), dim3(256), 0, s, q, epi);
}

// Pieces of the vocabulary: columns of one, and how many slices of K dx's product takes (one piece only)
struct Pieces { int64_t cols, count; int32_t slices; };
Pieces pieces_of(const DenseLogprobsParams &p)
{
    const int64_t e = (int64_t)esize(p), Mp = up(p.M, LINE / e);
    int64_t cols = p.piece_bytes / (Mp * e) / 256 * 256;
    if (cols < 256) cols = 256;
    if (cols > PIECE_MAX) cols = PIECE_MAX;
    Pieces k;
    k.count = (p.V + cols - 1) / cols;
    k.cols = up((p.V + k.count - 1) / k.count, 256);
    k.count = (p.V + k.cols - 1) / k.cols;
    k.slices = 1;
    const int64_t tiles = ((p.M + 127) / 128) * ((p.K + 127) / 128), lines = up(p.V, LINE / e) * e / LINE;
    if (k.count == 1 && tiles < 256) {
        int64_t n = 512 / tiles;
        if (n > lines / 8) n = lines / 8;
        if (n > 64) n = 64;
        k.slices = n < 1 ? 1 : (int32_t)n;
        const int64_t each = (lines + k.slices - 1) / k.slices;       // no slice is empty
        k.slices = (int32_t)((lines + each - 1) / each);
    }
    return k;
}

struct Layout { int64_t g, gt, wt, xt, acc, bytes; };
Layout layout_of(const DenseLogprobsParams &p, const Pieces &k)
{
    const int64_t e = (int64_t)esize(p), Mp = up(p.M, LINE / e);
    Layout l;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
    l.g = take(p.M * k.cols * e);
    l.gt = take(k.cols * Mp * e);
    l.wt = take(p.K * k.cols * e);
    l.xt = take(p.K * Mp * e);
    l.acc = take(k.count > 1 || k.slices > 1 ? (int64_t)k.slices * p.M * p.K * 4 : 0);
    l.bytes = at;
    return l;
}

template <typename E> hipError_t forward(const DenseLogprobsParams &p, hipStream_t s)
{
    NtParams q{};
    q.x = p.x; q.w = p.w; q.M = p.M; q.N = p.V; q.ldx = p.ldx; q.ldw = p.ldw; q.kbytes = (int32_t)up(p.K * sizeof(E), 16);
    const int32_t tiles = (int32_t)((p.V + 127) / 128);
    StatsEpi epi{};
    epi.part = (float2 *)p.part; epi.hit = (float *)p.part + 2 * (int64_t)tiles * p.M; epi.tok = p.tok; epi.M = p.M; epi.V = p.V;
    go_nt<E>(q, epi, 1, s);
    hipError_t er = hipGetLastError();
    if (er != hipSuccess) return er;
    hipLaunchKernelGGL(dense_logprobs_join_kernel, dim3((unsigned)((p.M + 31) / 32)), dim3(256), 0, s, epi.part, epi.hit, p.tok, p.lp, p.lse, p.M, p.V, tiles);
    return hipGetLastError();
}

template <typename E> void turn(const void *src, void *dst, int64_t R, int64_t C, int64_t ld, int64_t Rp, const DenseLogprobsParams *rows, hipStream_t s)
{
    hipLaunchKernelGGL((turn_rows_kernel<E>), dim3((unsigned)((Rp + 63) / 64), (unsigned)((C + 63) / 64)), dim3(256), 0, s, (const E *)src, (E *)dst, R, C, ld, Rp,
                       rows ? rows->tok : nullptr, rows ? rows->dlp : nullptr, rows ? rows->dlse : nullptr, rows ? rows->V : 0);
}

template <typename E> hipError_t gradient(const DenseLogprobsParams &p, hipStream_t s)
{
    constexpr int64_t e = sizeof(E);
    const Pieces k = pieces_of(p);
    const Layout at = layout_of(p, k);
    const int64_t Mp = up(p.M, LINE / e);
    char *const ws = (char *)p.part;
    E *const g = (E *)(ws + at.g), *const gt = (E *)(ws + at.gt), *const wt = (E *)(ws + at.wt), *const xt = (E *)(ws + at.xt);
    float *const acc = (float *)(ws + at.acc);
    turn<E>(p.x, xt, p.M, p.K, p.ldx / e, Mp, &p, s);
    for (int64_t i = 0; i < k.count; ++i) {
        const int64_t v0 = i * k.cols, cols = p.V - v0 < k.cols ? p.V - v0 : k.cols, Vp = up(cols, LINE / e);
        const char *const w = (const char *)p.w + v0 * p.ldw;
        turn<E>(w, wt, cols, p.K, p.ldw / e, Vp, nullptr, s);
        NtParams q{};
        q.x = p.x; q.w = w; q.M = Mp; q.N = Vp; q.ldx = p.ldx; q.ldw = p.ldw; q.kbytes = (int32_t)up(p.K * e, 16);
        GradEpi<E> ge{};
        ge.g = g; ge.gt = gt; ge.ldg = Vp; ge.ldgt = Mp; ge.tok = p.tok; ge.lse = p.lse_in; ge.dlp = p.dlp; ge.dlse = p.dlse;
        ge.M = p.M; ge.V = p.V; ge.v0 = v0; ge.Vp = Vp; ge.Mp = Mp;
        q.M = p.M; q.N = cols;                   // rows of x and w that are there; the tiles cover the padding behind them
        go_nt<E>(q, ge, 1, s);
        NtParams a{};
        a.x = g; a.w = wt; a.M = p.M; a.N = p.K; a.ldx = a.ldw = Vp * e; a.kbytes = (int32_t)(Vp * e);
        OutEpi o{};
        o.M = p.M; o.N = p.K; o.y = p.dx; o.y_dtype = p.dtype;
        if (k.slices > 1) {
            o.sum = acc;
        } else {
            o.before = i > 0 ? acc : nullptr;
            o.sum = i + 1 < k.count ? acc : nullptr;
        }
        go_nt<E>(a, o, k.slices, s);
        NtParams b{};
        b.x = gt; b.w = xt; b.M = cols; b.N = p.K; b.ldx = b.ldw = Mp * e; b.kbytes = (int32_t)(Mp * e);
        OutEpi d{};
        d.M = cols; d.N = p.K; d.y = (E *)p.dw + v0 * p.K; d.y_dtype = p.dtype;
        go_nt<E>(b, d, 1, s);
    }
    hipError_t er = hipGetLastError();
    if (er != hipSuccess || k.slices == 1) return er;
    SumShares q{};
    q.part = acc; q.P = k.slices; q.J = q.stride = p.M * p.K; q.dst = p.dx; q.dst_dtype = p.dtype;
    return launch_sum_shares(q, s);
}

}  // namespace

bool dense_logprobs_fits(const DenseLogprobsParams &p, bool grad)
{
    // a row's bytes, and those of a row of the transposed operands, are reached by 31-bit offsets from a tile's first row
    if (p.M < 1 || p.V < 1 || p.K < 1 || p.M > DENSE_LOGPROBS_MAX_ROWS || p.V > 0x7fffffff || p.K > DENSE_LOGPROBS_MAX_K) return false;
    if (!launch_has(((p.M + 127) / 128) * ((p.V + 127) / 128), 256)) return false;
    return !grad || (p.M * p.K + 63) / 64 <= 0x3fffff;
}

int64_t dense_logprobs_part_bytes(const DenseLogprobsParams &p, bool grad)
{
    if (!grad) return (2 * ((p.V + 127) / 128) + 1) * p.M * 4;
    return layout_of(p, pieces_of(p)).bytes;
}

hipError_t launch_dense_logprobs(const DenseLogprobsParams &p, hipStream_t s)
{
    if (!dense_logprobs_fits(p, false) || !p.part || p.ldx % 16 != 0 || p.ldw % 16 != 0) return hipErrorInvalidValue;
    return p.dtype == DT_BF16 ? forward<uint16_t>(p, s) : forward<float>(p, s);
}

hipError_t launch_dense_logprobs_grad(const DenseLogprobsParams &p, hipStream_t s)
{
    if (!dense_logprobs_fits(p, true) || !p.part || p.ldx % 16 != 0 || p.ldw % 16 != 0) return hipErrorInvalidValue;
    return p.dtype == DT_BF16 ? gradient<uint16_t>(p, s) : gradient<float>(p, s);
}

}  // namespace rl

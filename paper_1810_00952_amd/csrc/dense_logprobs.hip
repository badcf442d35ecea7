// Token log probabilities over a large vocabulary, from the last layer's rows x[M, K] and the vocabulary's w[V, K], and their gradients, without
// the logits l = x w^T in memory:
//
//   lse = ln sum_v e^l,  lp = l[tok] - lse;   dl = dlp (1[v = tok] - p) + dlse p,  p = e^(l - lse);   dx = dl w,  dw = dl^T x
//
// Forward: a product's tile leaves a maximum and a sum of exponentials a row, and the token's logit where it is its column; a second launch joins
// them.  Gradient, for pieces of the vocabulary: the piece's logits once more, dl from them, rounded to x's type as a product's operand and stored
// as it lies and transposed; then dx += dl w and dw = dl^T x in one launch, all three products of rows that lie along the contraction.  x and w are
// transposed for the last two.  Of up to sixteen rows both gradients are one pass over w.
//
// The matrix pipes bound it, few rows HBM.  bf16: 8192 x 50001 x 1024 the logits 728 to 752 us (1.13 PF/s), seven pieces of dl 160 each, of both gradients 205
// (1.17 PF/s); 4096 x 32000 x 1024 forward 246 (1.09); 8 x 131072 x 1024 50 (5.4 TB/s of w).  The pipes are busy 58 % of the cycles, at 1.6 to 1.9 GHz.
// f32: 777 x 10007 x 515 logits 77 (104 TF/s), dl 84, gradients 167.
#include "igemm_lds.h"

namespace rl {

namespace {

struct NtParams {                             // c[m, n] = sum_k x[m, k] w[n, k]; rows ldx, ldw bytes apart, kbytes of them (multiples of 16) count
    const void *x, *w;
    int64_t M, N, ldx, ldw;
    int32_t kbytes;
    int32_t nblk_m, nblk_n, nk;               // tiles along x and w, 128-byte lines of a row
    int32_t split_lines;                      // lines of a slice of K
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

// ---- what becomes of a tile's sums --------------------------------------------------------------------------------------------
// lds, a unit, is the workgroup's; own, TM times 4 KB of another, the wave's.  A lane has row m of x and, of every 32 of w's rows from n on, those at
// 8 k + 4 (its half of the wave) + i, k, i < 4.

// n .. n + 31 of row m as bf16, 16 bytes at a time: the halves of the wave swap what they hold of eight columns
__device__ __forceinline__ void put_row(uint16_t *to, const uint32_t (&c)[4][2], int half, bool in, int64_t n, int64_t N)
{
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4 out;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const auto got = __builtin_amdgcn_permlane32_swap(c[2 * h][d], c[2 * h + 1][d], false, false);
            out[d] = got[0]; out[2 + d] = got[1];
        }
        const int at = 16 * h + 8 * half;
        if (in && n + at < N) *(u32x4 *)(to + at) = out;
    }
#endif
}

// the rows' maxima and sums of exponentials over the tile's columns, and the tokens' logits
struct StatsEpi {
    float2 *part; float *hit; const int32_t *tok; int64_t M, V;

    // WN waves' maxima and sums meet in `lds`
    template <int WM, int WN, int TM, int TN> __device__ __forceinline__ void operator()(f32x16 (&acc)[TM][TN], int64_t m0, int64_t n0, int32_t bn, int wm, int wn, unsigned char *lds, unsigned char *own) const
    {
        constexpr int BM = WM * TM * 32;
        const int lane = threadIdx.x & 63, frow = lane & 31, half = lane >> 5;
        Soft *const seen = (Soft *)lds;                             // [WN][BM]
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + (wm * TM + i) * 32 + frow;
            const int32_t at = m < M ? tok[m] : -1;
            Soft s{-INFINITY, 0.0f};
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t nj = n0 + (wn * TN + j) * 32;
                if (nj + 32 > V) {                                  // columns behind the last
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        if (nj + 4 * half + 8 * (q >> 2) + (q & 3) >= V) acc[i][j][q] = -INFINITY;
                }
                const int64_t rel = at - nj - 4 * half;            // of the lane's columns: bit 2 clear, below 32
                if (at >= 0 && at < V && rel >= 0 && rel < 32 && (rel & 4) == 0) {
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        if (rel == 8 * (q >> 2) + (q & 3)) hit[m] = acc[i][j][q];
                }
#pragma unroll
                for (int q = 0; q < 16; ++q) s.m = fmaxf(s.m, acc[i][j][q]);
            }
            // of NaN a maximum is the other number: the sum has it
            const float top = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) s.s += __expf(acc[i][j][q] - top);
            Soft o{__shfl_xor(s.m, 32), __shfl_xor(s.s, 32)};
            s = join(s, o);
            if (half == 0) seen[wn * BM + (wm * TM + i) * 32 + frow] = s;
        }
        __syncthreads();
        for (int r = threadIdx.x; r < BM; r += 64 * WM * WN) {
            if (m0 + r >= M) break;
            Soft s = seen[r];
#pragma unroll
            for (int w = 1; w < WN; ++w) s = join(s, seen[w * BM + r]);
            part[(int64_t)bn * M + m0 + r] = float2{s.m, s.s};
        }
    }
};

// dl to g, as it lies, where there is one, and to gt, transposed
template <typename E> struct GradEpi {
    E *g, *gt; int64_t ldg, ldgt;             // elements
    const int32_t *tok; const float *lse, *dlp, *dlse;
    int64_t M, V, v0, Vp, Mp;                 // columns v0 .. of the vocabulary; Vp of them are written, Mp rows: multiples of 128 bytes

    template <int WM, int WN, int TM, int TN> __device__ __forceinline__ void operator()(f32x16 (&acc)[TM][TN], int64_t m0, int64_t n0, int32_t, int wm, int wn, unsigned char *lds, unsigned char *own) const
    {
        const int lane = threadIdx.x & 63, frow = lane & 31, half = lane >> 5;
        float end[TM], one[TM], all[TM];      // lse, dlp, dlse - dlp of the lane's rows
        int32_t at[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + (wm * TM + i) * 32 + frow;
            const bool in = m < M;
            at[i] = in ? tok[m] : -1;
            const bool given = at[i] >= 0 && at[i] < V;
            end[i] = in ? lse[m] : 0.0f;
            if (end[i] == -INFINITY) end[i] = INFINITY;            // of no logits: p is 0
            one[i] = in && given ? dlp[m] : 0.0f;
            all[i] = in ? dlse[m] - one[i] : 0.0f;
        }
        constexpr int ROW = TM * 64 + 32;     // bytes of a row of the transposed block in LDS, 32 behind its 32 TM bf16: rows begin at other banks
        static_assert(32 * ROW <= TM * 4096, "the wave's own part of LDS");
        unsigned char *const block = own;
        const int64_t mw = m0 + wm * TM * 32;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t nj = n0 + (wn * TN + j) * 32;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int64_t m = mw + i * 32 + frow;
                const bool none = one[i] == 0.0f && all[i] == 0.0f;
                const int64_t rel = at[i] - v0 - nj - 4 * half;
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int col = 8 * (q >> 2) + (q & 3);
                    const float v = __builtin_fmaf(all[i], __expf(acc[i][j][q] - end[i]), rel == col ? one[i] : 0.0f);
                    acc[i][j][q] = none || v0 + nj + 4 * half + col >= V ? 0.0f : v;
                }
                if constexpr (sizeof(E) == 4) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int64_t n = nj + 8 * k + 4 * half;
                        const f32x4 v = {acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]};
                        if (n < Vp) {
                            if (g && m < M) *(f32x4 *)(g + m * ldg + n) = v;
                            if (m < Mp) {
#pragma unroll
                                for (int c = 0; c < 4; ++c) gt[(n + c) * ldgt + m] = v[c];
                            }
                        }
                    }
                } else {
                    uint32_t c[4][2];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int d = 0; d < 2; ++d) c[k][d] = pack_bf16x2(acc[i][j][4 * k + 2 * d], acc[i][j][4 * k + 2 * d + 1]);
                    // two rows' numbers of one column are a word of the transposed block: an even lane takes the first of two columns, an odd one the other
                    const bool odd = lane & 1;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int d = 0; d < 2; ++d) {
                            const uint32_t mine = c[k][d], other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, 0xb1, 0xf, 0xf, true);
                            const uint32_t word = odd ? (other >> 16) | (mine & 0xffff0000u) : (mine & 0xffffu) | (other << 16);
                            *(uint32_t *)(block + (8 * k + 4 * half + 2 * d + (odd ? 1 : 0)) * ROW + i * 64 + (frow & 30) * 2) = word;
                        }
                    put_row((uint16_t *)g + m * ldg + nj, c, half, g && m < M, nj, Vp);
                }
            }
            if constexpr (sizeof(E) == 2) {
                wave_lds_exchange();
                constexpr int PER = TM * 4;                         // 16-byte pieces of a row
#pragma unroll
                for (int r = 0; r < 32 * PER / 64; ++r) {
                    const int q = r * 64 + lane, n = q / PER, c = q % PER;
                    const u32x4 v = *(const u32x4 *)(block + n * ROW + c * 16);
                    if (nj + n < Vp && mw + c * 8 < Mp) *(u32x4 *)(gt + (nj + n) * ldgt + mw + c * 8) = v;
                }
                wave_lds_exchange();
            }
        }
    }
};

// c (+ what was added up before) to y or, of a slice of K, to its share
struct OutEpi {
    void *y; const float *before; float *sum;  // sum: f32, in place of y
    int64_t M, N; int32_t y_dtype;

    template <int WM, int WN, int TM, int TN> __device__ __forceinline__ void operator()(f32x16 (&acc)[TM][TN], int64_t m0, int64_t n0, int32_t, int wm, int wn, unsigned char *, unsigned char *) const
    {
        const int lane = threadIdx.x & 63, frow = lane & 31, half = lane >> 5;
        const bool fours = N % 4 == 0, eights = N % 8 == 0;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t m = m0 + (wm * TM + i) * 32 + frow;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t nj = n0 + (wn * TN + j) * 32;
                f32x4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[k] = f32x4{acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]};
                    const int64_t n = nj + 8 * k + 4 * half, to = m * N + n;
                    if (before && m < M) {
                        if (fours) {
                            if (n < N) v[k] += *(const f32x4 *)(before + to);
                        } else {
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                if (n + c < N) v[k][c] += before[to + c];
                        }
                    }
                }
                if (!sum && y_dtype == DT_BF16 && eights) {
                    uint32_t c[4][2];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int d = 0; d < 2; ++d) c[k][d] = pack_bf16x2(v[k][2 * d], v[k][2 * d + 1]);
                    put_row((uint16_t *)y + m * N + nj, c, half, m < M, nj, N);
                    continue;
                }
                if (m >= M) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t n = nj + 8 * k + 4 * half, to = m * N + n;
                    if (fours && (sum || y_dtype != DT_BF16)) {
                        if (n < N) *(f32x4 *)((sum ? sum : (float *)y) + to) = v[k];
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (n + c < N) store_from_f32(sum ? (void *)sum : y, sum ? DT_F32 : y_dtype, to + c, v[k][c]);
                    }
                }
            }
        }
    }
};

}  // namespace

// ---------------------------------------------------------------------------
// WM x WN waves, each TM x TN groups of 32 rows of x and of w
// ---------------------------------------------------------------------------
template <typename E, int WM, int WN, int TM, int TN, typename Epi>
__device__ __forceinline__ void nt_tile(const NtParams &p, const Epi &epi, int32_t block, int32_t slice)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, W = WM * WN, UNIT = BM * 128;
    constexpr int XL = BM / 8 / W, LPT = 2 * XL;                   // direct loads per wave: of a unit, of a line of both
    static_assert(BM == BN && (BM / 8) % W == 0, "lines of x and of w take one unit each, in whole loads of every wave's");
    // arrays of their own: of requests into one the compiler would make every read wait
    __shared__ __attribute__((aligned(1024))) unsigned char st0[UNIT];
    __shared__ __attribute__((aligned(1024))) unsigned char st1[UNIT];
    __shared__ __attribute__((aligned(1024))) unsigned char st2[UNIT];
    __shared__ __attribute__((aligned(1024))) unsigned char st3[UNIT];
    __shared__ __attribute__((aligned(1024))) unsigned char st4[UNIT];

    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // each XCD a contiguous run of tiles; inside a run, column tiles in groups of eight with the row tiles fastest
    int32_t bm, bn;
    {
        constexpr int GN = 8;
        const int32_t bid = xcd_run(block, p.nblk_m * p.nblk_n), grp = bid / (GN * p.nblk_m), within = bid - grp * GN * p.nblk_m;
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
    const int32_t begin = slice * p.split_lines, end = min(begin + p.split_lines, p.nk), lines = end - begin;
    // the d-th load of a line of x or w into a unit; behind the last line: zeros
    auto dma = [&](unsigned char *to, bool w, int32_t line, int d) {
        const int i = w ? XL + d : d;
        const int32_t at = (begin + line) * 128;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(w ? rw : rx, RL_LDS_PTR(to + (wave * XL + d) * 1024), 16, line < lines && at < room[i] ? voff[i] + at : OOB, 0, 0, 0);
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
    auto fragments = [&](const unsigned char *x, const unsigned char *w, int ks) {
#pragma unroll
        for (int j = 0; j < TN; ++j) fw[ks & 1][j] = *(const u32x4 *)(w + (wn * TN + j) * 4096 + f_off[ks]);
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[ks & 1][i] = *(const u32x4 *)(x + (wm * TM + i) * 4096 + f_off[ks]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // a k-step's MFMAs; to: a unit's requests between them
    auto multiply = [&](int ks, unsigned char *to, bool w, int32_t line) {
        constexpr int N = TM * TN;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                Mfma<E>::go(acc[i][j], fw[ks & 1][j], fx[ks & 1][i]);
                if (to) {
                    const int n = i * TN + j;
#pragma unroll
                    for (int d = n * XL / N; d < (n + 1) * XL / N; ++d) dma(to, w, line, d);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    // Line t of x in x0, of w in w0; the next ones in x1 and w1, of which w's is under way; x's of the line after that goes where w's of the line
    // before was, w's of it to x0, which is free from the barrier on: the last k-step's fragments are in registers by then.
    int32_t t_ = 0;
    auto body = [&](unsigned char *x0, unsigned char *w0, unsigned char *x1, unsigned char *w1, unsigned char *x2) {
        fragments(x0, w0, 1);
        multiply(0, x2, false, t_ + 2);
        fragments(x0, w0, 2);
        multiply(1, nullptr, false, 0);
        fragments(x0, w0, 3);
        multiply(2, nullptr, false, 0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(XL) : "memory");
        fragments(x1, w1, 0);
        multiply(3, x0, true, t_ + 2);
        ++t_;
    };
#pragma unroll
    for (int d = 0; d < XL; ++d) dma(st0, false, 0, d);
#pragma unroll
    for (int d = 0; d < XL; ++d) dma(st1, true, 0, d);
#pragma unroll
    for (int d = 0; d < XL; ++d) dma(st2, false, 1, d);
#pragma unroll
    for (int d = 0; d < XL; ++d) dma(st3, true, 1, d);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(2 * XL) : "memory");
    fragments(st0, st1, 0);
    // item k of x0, w0, x1, w1, .. is in unit k % 5
#pragma unroll 1
    while (t_ + 5 <= lines) {
        body(st0, st1, st2, st3, st4);
        body(st2, st3, st4, st0, st1);
        body(st4, st0, st1, st2, st3);
        body(st1, st2, st3, st4, st0);
        body(st3, st4, st0, st1, st2);
    }
    if (t_ < lines) body(st0, st1, st2, st3, st4);
    if (t_ < lines) body(st2, st3, st4, st0, st1);
    if (t_ < lines) body(st4, st0, st1, st2, st3);
    if (t_ < lines) body(st1, st2, st3, st4, st0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");      // the trailing requests; from here the units are free

    // a wave's own part: half of a unit where there are eight waves, else a unit
    constexpr int SHARE = W > 4 ? 2 : 1;
    unsigned char *const unit = wave / SHARE == 0 ? st1 : wave / SHARE == 1 ? st2 : wave / SHARE == 2 ? st3 : st4;
    static_assert(UNIT / SHARE >= TM * 4096 && WN * BM * sizeof(Soft) <= UNIT, "what an epilogue wants is there");
    epi.template operator()<WM, WN, TM, TN>(acc, m0, n0, bn, wm, wn, st0, unit + wave % SHARE * (UNIT / SHARE));
#endif
}

template <typename E, int WM, int WN, int TM, int TN, typename Epi>
__global__ __launch_bounds__(64 * WM * WN) void nt_tile_kernel(const NtParams p, const Epi epi)
{
    nt_tile<E, WM, WN, TM, TN>(p, epi, blockIdx.x, 0);
}

// dx's product and dw's, the slices of K of each one behind the other
template <typename E, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void nt_pair_kernel(const NtParams a, const OutEpi ea, int32_t slices_a, const NtParams b, const OutEpi eb)
{
    const int32_t of_a = a.nblk_m * a.nblk_n, bid = (int32_t)blockIdx.x;
    const bool first = bid < of_a * slices_a;
    const NtParams p = first ? a : b;
    OutEpi e = first ? ea : eb;
    const int32_t at = first ? bid : bid - of_a * slices_a, tiles = p.nblk_m * p.nblk_n, slice = at / tiles;
    if (e.sum) e.sum += (int64_t)slice * e.M * e.N;
    if (e.before) e.before += (int64_t)slice * e.M * e.N;
    nt_tile<E, WM, WN, TM, TN>(p, e, at - slice * tiles, slice);
}

// ---------------------------------------------------------------------------
// rows' sums of all tiles; ROWS rows a workgroup, 1024 / ROWS threads a row
// ---------------------------------------------------------------------------
template <int ROWS>
__global__ __launch_bounds__(1024) void dense_logprobs_join_kernel(const float2 *part, const float *hit, const int32_t *tok, float *lp, float *lse, int64_t M, int64_t V, int32_t tiles)
{
    constexpr int SHARES = 1024 / ROWS;
    __shared__ Soft seen[SHARES][ROWS];
    const int r = threadIdx.x % ROWS, share = threadIdx.x / ROWS;
    const int64_t m = (int64_t)blockIdx.x * ROWS + r;
    Soft s{-INFINITY, 0.0f};
    if (m < M) {
#pragma unroll 4
        for (int32_t t = share; t < tiles; t += SHARES) {
            const float2 v = part[(int64_t)t * M + m];
            s = join(s, Soft{v.x, v.y});
        }
    }
    seen[share][r] = s;
    __syncthreads();
#pragma unroll
    for (int n = SHARES / 2; n > 0; n /= 2) {
        if (share < n) {
            s = join(s, seen[share + n][r]);
            seen[share][r] = s;
        }
        __syncthreads();
    }
    if (share == 0 && m < M) {
        const float all = s.m == INFINITY ? __uint_as_float(0x7fc00000u) : s.m + __logf(s.s);
        const int32_t at = tok[m];
        lse[m] = all;
        lp[m] = at < 0 || at >= V ? 0.0f : all == -INFINITY ? -INFINITY : hit[m] - all;
    }
}

// whether a row has a derivative; what stands in one without reaches nothing
__device__ __forceinline__ bool takes_part(const int32_t *tok, const float *dlp, const float *dlse, int64_t m, int64_t V)
{
    const int32_t k = tok[m];
    return dlse[m] != 0.0f || (k >= 0 && k < V && dlp[m] != 0.0f);
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
            if (tok) part = takes_part(tok, dlp, dlse, r0 + r, V);
            if (part) v = src[(r0 + r) * ld + c0 + c];
        }
        s[r][c] = v;
    }
    __syncthreads();
    for (int k = w; k < 64; k += 4)
        if (c0 + k < C && r0 + c < Rp) dst[(c0 + k) * Rp + r0 + c] = s[c][k];
}

// ---------------------------------------------------------------------------
// Both gradients of up to MR rows: a lane has VEC columns of all of them, reads w's rows as they lie and writes dw's, with the wave's numbers of dl; grid's
// y: slices of w's rows, of which each wave takes every fourth and whose dx are added up behind.  The products' way would turn w first, two passes more
// over it, and multiply tiles of 64 rows.  HBM bounds it: f32 5 x 44311 x 3144 240 us (w read, dw written: 4.6 TB/s; logits and gradients together
// 954 -> 569), bf16 3 x 24355 x 2240 46 (175 -> 94).  Of more rows the vector units would: sixteen are 32 operations a number of w.
// ---------------------------------------------------------------------------
template <typename E, int MR> struct Few {
    static constexpr int VEC = sizeof(E) == 2 && MR < 16 ? 8 : 4, WORDS = VEC * (int)sizeof(E) / 4, WIDE = 64 * VEC;
    struct raw { uint32_t r[WORDS]; };
    static __device__ __forceinline__ raw load(const char *p)
    {
        raw q;
        if constexpr (WORDS == 4) {
            const u32x4 v = *(const u32x4 *)p;
#pragma unroll
            for (int c = 0; c < 4; ++c) q.r[c] = v[c];
        } else {
            const u32x2 v = *(const u32x2 *)p;
            q.r[0] = v[0]; q.r[1] = v[1];
        }
        return q;
    }
    static __device__ __forceinline__ void unpack(const raw &q, float (&x)[VEC])
    {
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            if constexpr (sizeof(E) == 4) x[c] = __uint_as_float(q.r[c]);
            else x[c] = __uint_as_float(c & 1 ? q.r[c >> 1] & 0xffff0000u : q.r[c >> 1] << 16);
        }
    }
    // whole vectors, which need not lie at their size's multiple, and the row's last elements
    static __device__ __forceinline__ void store(E *p, const float (&x)[VEC], int64_t left)
    {
        typedef u32x4 u32x4_any __attribute__((aligned(2)));
        typedef u32x2 u32x2_any __attribute__((aligned(2)));
        uint32_t q[WORDS];
#pragma unroll
        for (int c = 0; c < WORDS; ++c) {
            if constexpr (sizeof(E) == 4) q[c] = __float_as_uint(x[c]);
            else q[c] = pack_bf16x2(x[2 * c], x[2 * c + 1]);
        }
        if (left >= VEC) {
            if constexpr (WORDS == 4) *(u32x4_any *)p = u32x4{q[0], q[1], q[2], q[3]};
            else *(u32x2_any *)p = u32x2{q[0], q[1]};
        } else {
#pragma unroll
            for (int c = 0; c < VEC; ++c)
                if (c < left) store_from_f32(p, sizeof(E) == 4 ? DT_F32 : DT_BF16, c, x[c]);
        }
    }
};

template <typename E, int MR>
__global__ __launch_bounds__(256) void few_rows_kernel(const uint32_t *__restrict__ gt, int64_t ldgt, const char *__restrict__ w, int64_t ldw, const char *__restrict__ x, int64_t ldx, const int32_t *tok, const float *dlp,
                                                       const float *dlse, const float *before, float *sum, E *dw, int32_t M, int64_t V, int64_t K, int64_t rows, int64_t slice_rows)
{
    typedef Few<E, MR> F;
    constexpr int VEC = F::VEC, WIDE = F::WIDE, UNDER_WAY = 8;
    __shared__ float s[MR][WIDE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t k0 = (int64_t)blockIdx.x * WIDE, k = k0 + lane * VEC;
    const int64_t begin = (int64_t)blockIdx.y * slice_rows, end = min(begin + slice_rows, rows);
    const int64_t left = K - k, at_k = (left > 0 ? k : 0) * (int64_t)sizeof(E);         // a lane behind the last column: the first one's, of which nothing is stored
    float acc[MR][VEC], xs[MR][VEC];
#pragma unroll
    for (int m = 0; m < MR; ++m) {
        typename F::raw q{};
        if (m < M && takes_part(tok, dlp, dlse, m, V)) q = F::load(x + m * ldx + at_k);
        F::unpack(q, xs[m]);
#pragma unroll
        for (int c = 0; c < VEC; ++c) acc[m][c] = 0.0f;
    }
    auto row = [&](const typename F::raw &q, int64_t v) __attribute__((always_inline)) {
        const uint32_t *const g = gt + v * ldgt;                     // words: of bf16 two rows' numbers
        float wv[VEC], d[VEC];
        F::unpack(q, wv);
#pragma unroll
        for (int c = 0; c < VEC; ++c) d[c] = 0.0f;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            float dl;
            if constexpr (sizeof(E) == 4) dl = __uint_as_float(g[m]);
            else dl = __uint_as_float(m & 1 ? g[m >> 1] & 0xffff0000u : g[m >> 1] << 16);
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                acc[m][c] = __builtin_fmaf(dl, wv[c], acc[m][c]);
                d[c] = __builtin_fmaf(dl, xs[m][c], d[c]);
            }
        }
        if (left > 0) F::store(dw + v * K + k, d, left);
    };
    const char *const from = w + at_k;
    int64_t v = begin + wave;
    for (; v + 4 * (UNDER_WAY - 1) < end; v += 4 * UNDER_WAY) {
        typename F::raw q[UNDER_WAY];
#pragma unroll
        for (int u = 0; u < UNDER_WAY; ++u) q[u] = F::load(from + (v + 4 * u) * ldw);
#pragma unroll
        for (int u = 0; u < UNDER_WAY; ++u) row(q[u], v + 4 * u);
    }
    for (; v < end; v += 4) row(F::load(from + v * ldw), v);
    for (int t = 0; t < 4; ++t) {                                    // the waves' sums, one behind the other
        if (wave == t) {
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
                for (int c = 0; c < VEC; ++c) s[m][lane * VEC + c] = t ? s[m][lane * VEC + c] + acc[m][c] : acc[m][c];
        }
        __syncthreads();
    }
    const int64_t share = (int64_t)blockIdx.y * M * K;
    for (int i = threadIdx.x; i < M * WIDE; i += 256) {
        const int m = i / WIDE, c = i % WIDE;
        if (k0 + c >= K) continue;
        const int64_t at = share + m * K + k0 + c;
        sum[at] = before ? before[at] + s[m][c] : s[m][c];
    }
}

namespace {

constexpr int64_t FEW = 16;                   // rows whose gradients are few_rows_kernel's
// columns of one of its workgroups
int64_t few_wide(const DenseLogprobsParams &p) { return p.dtype == DT_BF16 && p.M <= 8 ? 512 : 256; }
constexpr int64_t LINE = 128, PIECE_MAX = 1 << 20;      // a piece's columns: a row of dl is reached by 31-bit offsets from its tile's first
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
size_t esize(const DenseLogprobsParams &p) { return p.dtype == DT_BF16 ? 2 : 4; }

// Which tile, by an estimate of the time: us per 128-byte line of K of a workgroup that is alone on its CU, and per line and 256 workgroups where there are more
// (measured on products of one and of many workgroups a CU; 256 x 256 against 128 x 128 for dl of the first case above 170 against 180 us)
struct Tile { int32_t side; float alone, share; };
constexpr Tile tiles_bf16[] = {{64, 0.70f, 0.25f}, {128, 0.95f, 0.62f}, {256, 1.60f, 2.00f}};
constexpr Tile tiles_f32[] = {{64, 1.00f, 0.50f}, {128, 3.60f, 1.85f}};
int64_t tiles_along(int64_t n, int64_t side) { return (n + side - 1) / side; }
template <typename E, typename F> void each_tile(const F &look)
{
    if constexpr (sizeof(E) == 2) for (const Tile &t : tiles_bf16) look(t);
    else for (const Tile &t : tiles_f32) look(t);
}
// of the product [M, N]
template <typename E> int32_t tile_of(int64_t M, int64_t N)
{
    int32_t best = 0;
    float least = INFINITY;
    each_tile<E>([&](const Tile &t) {
        const float line = fmaxf(t.alone, t.share * (float)(tiles_along(M, t.side) * tiles_along(N, t.side)) / 256.0f);
        if (line < least) { least = line; best = t.side; }
    });
    return best;
}

// Tile and slices of K of two products in one launch, dx [M, K] over `cols` and dw [cols, K] over M: a product of few long tiles is cut into slices near what
// a CU has of the whole, whose shares are written and read once more (f32 3519 x 7399 x 128 475 -> 131 us, bf16 1809 x 34304 x 869 709 -> 355)
struct Pair { int32_t side, a, b; };
template <typename E> Pair pair_of(int64_t M, int64_t K, int64_t cols, int64_t most_bytes)
{
    constexpr int64_t per = LINE / sizeof(E);
    Pair best{0, 1, 1};
    float least = INFINITY;
    each_tile<E>([&](const Tile &t) {
        const int64_t ta = tiles_along(M, t.side) * tiles_along(K, t.side), tb = tiles_along(cols, t.side) * tiles_along(K, t.side);
        const int64_t la = tiles_along(cols, per), lb = tiles_along(M, per);
        const float all = (float)(ta * la + tb * lb) / 256.0f;
        auto slices = [&](int64_t lines, int64_t bytes) {
            int64_t n = (int64_t)ceilf((float)lines / fmaxf(1.25f * all * t.share / t.alone, 8.0f));
            n = n > 64 ? 64 : n;
            if (n * bytes > most_bytes) n = most_bytes / bytes;
            return (int32_t)(n > 1 ? n : 1);
        };
        Pair f{t.side, slices(la, M * K * 4), slices(lb, cols * K * 4)};
        const float lines = fmaxf((float)la / f.a, (float)lb / f.b);
        const float shares = (f.a > 1 ? (float)f.a * M * K : 0.0f) + (f.b > 1 ? (float)f.b * cols * K : 0.0f);
        const float us = fmaxf(lines * t.alone, all * t.share) + shares * 8.0f / 5e6f;
        if (us < least) { least = us; best = f; }
    });
    return best;
}

void split(NtParams &q, int32_t side, int32_t slices)
{
    q.nblk_m = (int32_t)tiles_along(q.M, side);
    q.nblk_n = (int32_t)tiles_along(q.N, side);
    q.nk = (int32_t)((q.kbytes + LINE - 1) / LINE);
    q.split_lines = (q.nk + slices - 1) / slices;
}

template <typename E, typename Epi> void go_nt(NtParams q, const Epi &epi, int32_t side, hipStream_t s)
{
    split(q, side, 1);
    const dim3 grid((unsigned)((int64_t)q.nblk_m * q.nblk_n));
    if constexpr (sizeof(E) == 2) {
        if (side == 256) { hipLaunchKernelGGL((nt_tile_kernel<E, 2, 4, 4, 2, Epi>), grid, dim3(512), 0, s, q, epi); return; }
    }
    if (side == 128) hipLaunchKernelGGL((nt_tile_kernel<E, 2, 2, 2, 2, Epi>), grid, dim3(256), 0, s, q, epi);
    else hipLaunchKernelGGL((nt_tile_kernel<E, 2, 2, 1, 1, Epi>), grid, dim3(256), 0, s, q, epi);
}

template <typename E> void go_pair(NtParams a, const OutEpi &ea, NtParams b, const OutEpi &eb, const Pair &f, hipStream_t s)
{
    split(a, f.side, f.a);
    split(b, f.side, f.b);
    const dim3 grid((unsigned)((int64_t)a.nblk_m * a.nblk_n * f.a + (int64_t)b.nblk_m * b.nblk_n * f.b));
    if constexpr (sizeof(E) == 2) {
        if (f.side == 256) { hipLaunchKernelGGL((nt_pair_kernel<E, 2, 4, 4, 2>), grid, dim3(512), 0, s, a, ea, f.a, b, eb); return; }
    }
    if (f.side == 128) hipLaunchKernelGGL((nt_pair_kernel<E, 2, 2, 2, 2>), grid, dim3(256), 0, s, a, ea, f.a, b, eb);
    else hipLaunchKernelGGL((nt_pair_kernel<E, 2, 2, 1, 1>), grid, dim3(256), 0, s, a, ea, f.a, b, eb);
}

// Pieces of the vocabulary: columns of one, and how its gradients' products go
struct Pieces { int64_t cols, count; Pair pair; };
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
    const int64_t real = k.cols < p.V ? k.cols : p.V;
    if (p.M <= FEW) {
        // slices: two workgroups a CU
        const int64_t wide = tiles_along(p.K, few_wide(p)), most = (real + 63) / 64;
        int64_t n = 512 / wide > 1 ? 512 / wide : 1;
        if (n > most) n = most;
        k.pair = Pair{0, (int32_t)n, 1};
        return k;
    }
    k.pair = p.dtype == DT_BF16 ? pair_of<uint16_t>(p.M, p.K, real, p.piece_bytes) : pair_of<float>(p.M, p.K, real, p.piece_bytes);
    return k;
}

struct Layout { int64_t g, gt, wt, xt, dx, dw, bytes; };
Layout layout_of(const DenseLogprobsParams &p, const Pieces &k)
{
    const int64_t e = (int64_t)esize(p), Mp = up(p.M, LINE / e);
    Layout l;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
    const bool few = p.M <= FEW;
    l.g = take(few ? 0 : p.M * k.cols * e);
    l.gt = take(k.cols * Mp * e);
    l.wt = take(few ? 0 : p.K * k.cols * e);
    l.xt = take(few ? 0 : p.K * Mp * e);
    l.dx = take(few || k.count > 1 || k.pair.a > 1 ? (int64_t)k.pair.a * p.M * p.K * 4 : 0);
    l.dw = take(k.pair.b > 1 ? (int64_t)k.pair.b * k.cols * p.K * 4 : 0);
    l.bytes = at;
    return l;
}

template <typename E> hipError_t forward(const DenseLogprobsParams &p, hipStream_t s)
{
    NtParams q{};
    q.x = p.x; q.w = p.w; q.M = p.M; q.N = p.V; q.ldx = p.ldx; q.ldw = p.ldw; q.kbytes = (int32_t)up(p.K * sizeof(E), 16);
    const int32_t side = tile_of<E>(p.M, p.V), tiles = (int32_t)tiles_along(p.V, side);
    StatsEpi epi{};
    epi.part = (float2 *)p.part; epi.hit = (float *)p.part + 2 * (int64_t)tiles * p.M; epi.tok = p.tok; epi.M = p.M; epi.V = p.V;
    go_nt<E>(q, epi, side, s);
    hipError_t er = hipGetLastError();
    if (er != hipSuccess) return er;
    if (p.M >= 1024) hipLaunchKernelGGL((dense_logprobs_join_kernel<32>), dim3((unsigned)((p.M + 31) / 32)), dim3(1024), 0, s, epi.part, epi.hit, p.tok, p.lp, p.lse, p.M, p.V, tiles);
    else hipLaunchKernelGGL((dense_logprobs_join_kernel<4>), dim3((unsigned)((p.M + 3) / 4)), dim3(1024), 0, s, epi.part, epi.hit, p.tok, p.lp, p.lse, p.M, p.V, tiles);
    return hipGetLastError();
}

template <typename E> void turn(const void *src, void *dst, int64_t R, int64_t C, int64_t ld, int64_t Rp, const DenseLogprobsParams *rows, hipStream_t s)
{
    hipLaunchKernelGGL((turn_rows_kernel<E>), dim3((unsigned)((Rp + 63) / 64), (unsigned)((C + 63) / 64)), dim3(256), 0, s, (const E *)src, (E *)dst, R, C, ld, Rp,
                       rows ? rows->tok : nullptr, rows ? rows->dlp : nullptr, rows ? rows->dlse : nullptr, rows ? rows->V : 0);
}

// of a piece: `rows` of the vocabulary from the v0-th on
template <typename E> void few_rows(const DenseLogprobsParams &p, const E *gt, int64_t ldgt, int64_t v0, int64_t rows, int32_t slices, float *sum, hipStream_t s)
{
    const dim3 grid((unsigned)tiles_along(p.K, few_wide(p)), (unsigned)slices), wg(256);
    auto with = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, wg, 0, s, (const uint32_t *)gt, (int64_t)(ldgt * sizeof(E) / 4), (const char *)p.w + v0 * p.ldw, p.ldw, (const char *)p.x, p.ldx, p.tok, p.dlp, p.dlse,
                           v0 > 0 ? sum : nullptr, sum, (E *)p.dw + v0 * p.K, (int32_t)p.M, p.V, p.K, rows, (rows + slices - 1) / slices);
    };
    if (p.M <= 4) with(few_rows_kernel<E, 4>);
    else if (p.M <= 8) with(few_rows_kernel<E, 8>);
    else with(few_rows_kernel<E, 16>);
}

template <typename E> hipError_t gradient(const DenseLogprobsParams &p, hipStream_t s)
{
    constexpr int64_t e = sizeof(E);
    const Pieces k = pieces_of(p);
    const Layout at = layout_of(p, k);
    const int64_t Mp = up(p.M, LINE / e);
    char *const ws = (char *)p.part;
    E *const g = (E *)(ws + at.g), *const gt = (E *)(ws + at.gt), *const wt = (E *)(ws + at.wt), *const xt = (E *)(ws + at.xt);
    float *const of_x = (float *)(ws + at.dx), *const of_w = (float *)(ws + at.dw);
    SumShares sums{};
    sums.dst_dtype = p.dtype;
    const bool few = p.M <= FEW;
    if (!few) turn<E>(p.x, xt, p.M, p.K, p.ldx / e, Mp, &p, s);
    for (int64_t i = 0; i < k.count; ++i) {
        const int64_t v0 = i * k.cols, cols = p.V - v0 < k.cols ? p.V - v0 : k.cols, Vp = up(cols, LINE / e);
        const char *const w = (const char *)p.w + v0 * p.ldw;
        if (!few) turn<E>(w, wt, cols, p.K, p.ldw / e, Vp, nullptr, s);
        NtParams q{};
        q.x = p.x; q.w = w; q.M = p.M; q.N = cols; q.ldx = p.ldx; q.ldw = p.ldw; q.kbytes = (int32_t)up(p.K * e, 16);       // the tiles cover the padding of dl
        GradEpi<E> ge{};
        ge.g = few ? nullptr : g; ge.gt = gt; ge.ldg = Vp; ge.ldgt = Mp; ge.tok = p.tok; ge.lse = p.lse_in; ge.dlp = p.dlp; ge.dlse = p.dlse;
        ge.M = p.M; ge.V = p.V; ge.v0 = v0; ge.Vp = Vp; ge.Mp = Mp;
        go_nt<E>(q, ge, tile_of<E>(p.M, cols), s);
        if (few) {
            few_rows<E>(p, gt, Mp, v0, cols, k.pair.a, of_x, s);
            continue;
        }
        NtParams a{};
        a.x = g; a.w = wt; a.M = p.M; a.N = p.K; a.ldx = a.ldw = Vp * e; a.kbytes = (int32_t)(Vp * e);
        OutEpi o{};
        o.M = p.M; o.N = p.K; o.y = p.dx; o.y_dtype = p.dtype;
        // every slice adds up over the pieces
        o.before = i > 0 ? of_x : nullptr;
        o.sum = k.pair.a > 1 || i + 1 < k.count ? of_x : nullptr;
        NtParams b{};
        b.x = gt; b.w = xt; b.M = cols; b.N = p.K; b.ldx = b.ldw = Mp * e; b.kbytes = (int32_t)(Mp * e);
        OutEpi d{};
        d.M = cols; d.N = p.K; d.y = (E *)p.dw + v0 * p.K; d.y_dtype = p.dtype;
        d.sum = k.pair.b > 1 ? of_w : nullptr;
        go_pair<E>(a, o, b, d, k.pair, s);
        if (k.pair.b > 1) {
            sums.part = of_w; sums.P = k.pair.b; sums.J = sums.J1 = sums.stride = cols * p.K; sums.dst = d.y;
            const hipError_t er = launch_sum_shares(sums, s);
            if (er != hipSuccess) return er;
        }
    }
    hipError_t er = hipGetLastError();
    if (er != hipSuccess || (k.pair.a == 1 && !few)) return er;
    sums.part = of_x; sums.P = k.pair.a; sums.J = sums.J1 = sums.stride = p.M * p.K; sums.dst = p.dx;
    return launch_sum_shares(sums, s);
}

}  // namespace

bool dense_logprobs_fits(const DenseLogprobsParams &p)
{
    // a row's bytes, and those of a row of the transposed operands, are reached by 31-bit offsets from a tile's first row
    if (p.M < 1 || p.V < 1 || p.K < 1 || p.M > DENSE_LOGPROBS_MAX_ROWS || p.V > 0x7fffffff || p.K > DENSE_LOGPROBS_MAX_K) return false;
    return launch_has(((p.M + 63) / 64) * ((p.V + 63) / 64), 256);
}

int64_t dense_logprobs_part_bytes(const DenseLogprobsParams &p, bool grad)
{
    const int32_t side = p.dtype == DT_BF16 ? tile_of<uint16_t>(p.M, p.V) : tile_of<float>(p.M, p.V);
    if (!grad) return (2 * tiles_along(p.V, side) + 1) * p.M * 4;
    return layout_of(p, pieces_of(p)).bytes;
}

hipError_t launch_dense_logprobs(const DenseLogprobsParams &p, hipStream_t s)
{
    if (!dense_logprobs_fits(p) || !p.part || p.ldx % 16 != 0 || p.ldw % 16 != 0) return hipErrorInvalidValue;
    return p.dtype == DT_BF16 ? forward<uint16_t>(p, s) : forward<float>(p, s);
}

hipError_t launch_dense_logprobs_grad(const DenseLogprobsParams &p, hipStream_t s)
{
    if (!dense_logprobs_fits(p) || !p.part || p.ldx % 16 != 0 || p.ldw % 16 != 0) return hipErrorInvalidValue;
    return p.dtype == DT_BF16 ? gradient<uint16_t>(p, s) : gradient<float>(p, s);
}

}  // namespace rl

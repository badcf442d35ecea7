// Product of 8-bit integers with a scale per row of x and per row of w:
//
//   y[m, n] = sx[m] sw[n] sum_k x[m, k] w[n, k] + b[n],   the sum exact in 32 bits
//
// w's rows are the MFMA's rows, so that a lane holds one row of x and runs of four columns of y.  Zeros stand behind a row of w up to a
// multiple of 128 bytes, so what stands behind a row of x (the next row) does not count, and K is worked off in whole 128-byte lines.
//
// Two kernels.  dense_q8_tile: tiles of both operands through LDS, two stages of 128 bytes a row, requested by direct loads; a tile's
// barrier stands before the last of its four k-steps, whose fragments are in registers by then, so that the tile after the next is
// requested into the stage being left and the next tile's first fragments are read under that step's MFMAs.
// dense_q8_direct: for few rows of x, where the time is w's way from memory: fragments straight into registers, K over the
// eight waves of a workgroup (whole lines in turn), whose sums meet in LDS: every wave's loads are under way at once.
//
// 8192 x 8192 x 4096 269 us (2.04 Pop/s), 4096 x 4096 x 16384 240 us (2.29), a library product of 8-bit integers without scales 2.2: the MFMAs are busy 52 % of the
// cycles at some 1.9 GHz without conflicts in LDS; what takes the other half is not known.  All of a tile's requests in one k-step 281 us.
// Short rows: a workgroup does one tile, whose first requests and results stand alone: K = 1024, 4096 rows by 1024, 2048 and 32000 columns
// 0.77, 1.08 and 1.36 Pop/s.  8 x 4096 x 4096 6.4 us: a launch and a chain of latencies.
#include "igemm_lds.h"

namespace rl {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

namespace {

struct Q8Grid { int32_t nblk_m, nblk_n, nk; };       // tiles along x and w, 128-byte lines of a row

// y of row m, columns n .. n + 3 from their exact sums
struct Epi4 {
    f32x4 sw, b;
    __device__ __forceinline__ Epi4(const DenseQ8Params &p, int64_t n)
    {
        if (p.N % 4 == 0) {                               // n is a multiple of 4
            const int64_t c = n < p.N ? n : p.N - 4;
            sw = *(const f32x4 *)(p.sw + c);
            b = p.b ? *(const f32x4 *)(p.b + c) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t c = n + k < p.N ? n + k : p.N - 1;
            sw[k] = p.sw[c];
            b[k] = p.b ? p.b[c] : 0.0f;
        }
    }
    __device__ __forceinline__ f32x4 operator()(const i32x4 &sum, float sx) const
    {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __builtin_fmaf((float)sum[k] * sx, sw[k], b[k]);
        return v;
    }
};

// y[m, n .. n + 3], n a multiple of 4
__device__ __forceinline__ void store4(const DenseQ8Params &p, int64_t m, int64_t n, const f32x4 &v)
{
    if (p.N % 4 == 0) {
        if (p.y_dtype == DT_BF16) *(u32x2 *)((uint16_t *)p.y + m * p.N + n) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else *(f32x4 *)((float *)p.y + m * p.N + n) = v;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (n + k < p.N) store_from_f32(p.y, p.y_dtype, m * p.N + n + k, v[k]);
    }
}

}  // namespace

// ---------------------------------------------------------------------------
// MT x NT groups of 16 rows of x and of w, all of K over eight waves
// ---------------------------------------------------------------------------
template <int MT, int NT>
__global__ __launch_bounds__(512) void dense_q8_direct_kernel(const DenseQ8Params p, const Q8Grid g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int W = 8, DEPTH = MT + NT > 4 ? 1 : MT + NT > 3 ? 2 : 3;              // lines a wave has under way beside the one it multiplies
    __shared__ i32x4 sums[W][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    const int32_t bm = blockIdx.x % g.nblk_m, bn = blockIdx.x / g.nblk_m;
    const int64_t m0 = (int64_t)bm * 16 * MT, n0 = (int64_t)bn * 16 * NT;
    // x is read to its last row's end (the lines behind it are zeros), w's rows are whole lines
    const int64_t xroom = (p.M - m0) * p.ldx;
    const rsrc_t rx = make_rsrc(p.x + m0 * p.ldx, (uint32_t)(xroom < 0x7fffffff ? xroom : 0x7fffffff));
    uint32_t xo[MT];
    const int8_t *wo[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) xo[i] = (uint32_t)((m0 + 16 * i + r < p.M ? 16 * i + r : p.M - 1 - m0) * p.ldx) + 16 * q;
#pragma unroll
    for (int j = 0; j < NT; ++j) wo[j] = p.w + (n0 + 16 * j + r < p.N ? n0 + 16 * j + r : p.N - 1) * p.ldw + 16 * q;

    i32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    i32x4 fx[DEPTH + 1][2][MT], fw[DEPTH + 1][2][NT];
    auto request = [&](int s, int32_t line) {
        const uint32_t at = (uint32_t)line * 128u;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < NT; ++j) fw[s][h][j] = *(const i32x4 *)(wo[j] + at + 64 * h);
#pragma unroll
            for (int i = 0; i < MT; ++i) fx[s][h][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, xo[i] + at + 64 * h, 0, 0));
        }
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[s][h][j], fx[s][h][i], acc[i][j], 0, 0, 0);
    };
    const int32_t mine = (g.nk - wave + W - 1) / W;                // lines wave, wave + 8, ...
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < mine) request(d, wave + d * W);
    int32_t k = 0;
    for (; k + DEPTH + 1 <= mine; k += DEPTH + 1) {
#pragma unroll
        for (int d = 0; d <= DEPTH; ++d) {
            if (k + d + DEPTH < mine) request((d + DEPTH) % (DEPTH + 1), wave + (k + d + DEPTH) * W);
            multiply(d);
        }
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (k + d < mine) multiply(d);

#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    // a group of sixteen rows of each a wave: lane's row of x is r, its columns 4 q .. 4 q + 3
    for (int t = wave; t < MT * NT; t += W) {
        i32x4 sum = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += sums[w][t][lane];
        const int64_t m = m0 + 16 * (t / NT) + r, n = n0 + 16 * (t % NT) + 4 * q;
        if (m < p.M && n < p.N) store4(p, m, n, Epi4(p, n)(sum, p.sx[m]));
    }
#endif
}

// ---------------------------------------------------------------------------
// WM x WN waves, each TM x TN groups of 32 rows of x and of w
// ---------------------------------------------------------------------------
template <int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void dense_q8_tile_kernel(const DenseQ8Params p, const Q8Grid g)
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
        const int32_t bid = xcd_run(blockIdx.x, g.nblk_m * g.nblk_n), grp = bid / (GN * g.nblk_m), within = bid - grp * GN * g.nblk_m;
        const int32_t gw = min(GN, g.nblk_n - grp * GN);
        bm = within / gw; bn = grp * GN + (within - bm * gw);
    }
    const int64_t m0 = (int64_t)bm * BM, n0 = (int64_t)bn * BN;
    // from the tile's first rows on: offsets stay small whatever the matrices' sizes
    const int64_t xroom = min((p.M - m0) * p.ldx, (int64_t)0x7fffffff), wroom = min((p.N - n0) * p.ldw, (int64_t)0x7fffffff);
    const rsrc_t rx = make_rsrc(p.x + m0 * p.ldx, (uint32_t)xroom), rw = make_rsrc(p.w + n0 * p.ldw, (uint32_t)wroom);

    // lane l of a load fills row l >> 3, position l & 7 of eight rows of 128 bytes; chunks of 16 swizzled by the row
    uint32_t voff[LPT];
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
        const bool x = i < XL;
        const int row = x ? (wave * XL + i) * 8 + (lane >> 3) : (wave * (LPT - XL) + i - XL) * 8 + (lane >> 3);
        const int chunk = (lane & 7) ^ ((row >> 1) & 7);
        const bool in = x ? m0 + row < p.M : n0 + row < p.N;
        voff[i] = in ? (uint32_t)row * (uint32_t)(x ? p.ldx : p.ldw) + chunk * 16 : OOB;
    }
    int32_t f_kt = 0;
    uint32_t f_at = 0;
    bool f_live = true;
    auto begin = [&]() { f_live = f_kt < g.nk; f_at = f_live ? (uint32_t)f_kt * 128u : 0u; ++f_kt; };
    auto dma = [&](unsigned char *st, int d) {
        unsigned char *to = d < XL ? st + (wave * XL + d) * 1024 : st + X_BYTES + (wave * (LPT - XL) + d - XL) * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d < XL ? rx : rw, RL_LDS_PTR(to), 16, f_live && voff[d] != OOB ? voff[d] + f_at : OOB, 0, 0, 0);
    };

    i32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;
    const int frow = lane & 31, fhalf = lane >> 5;
    int f_off[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) f_off[ks] = frow * 128 + (((2 * ks + fhalf) ^ ((frow >> 1) & 7)) << 4);
    i32x4 fw[2][TN], fx[2][TM];
    auto fragments = [&](const unsigned char *st, int ks) {
#pragma unroll
        for (int j = 0; j < TN; ++j) fw[ks & 1][j] = *(const i32x4 *)(st + X_BYTES + (wn * TN + j) * 4096 + f_off[ks]);
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[ks & 1][i] = *(const i32x4 *)(st + (wm * TM + i) * 4096 + f_off[ks]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // a k-step's MFMAs; req 0, 1: the first, second half of a tile's direct loads between them, 2: none
    auto multiply = [&](int ks, unsigned char *to, int req) {
        constexpr int HALF = LPT / 2, N = TM * TN;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[ks & 1][j], fx[ks & 1][i], acc[i][j], 0, 0, 0);
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
    for (; kt + 2 <= g.nk; kt += 2) {
        body(st0, st1);
        body(st1, st0);
    }
    if (kt < g.nk) body(st0, st1);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");      // the trailing requests; from here the stages are free

    // lane's row of x is frow, its columns 8 q + 4 fhalf .. + 3: bf16 of whole lines straight from registers, the rest through LDS, 4 KB of it a
    // wave's own, to whole lines of y
    static_assert(W * 4096 <= STAGE, "every wave's part is in the first stage");
    float *const park = (float *)st0 + wave * 1024;
    const bool whole = p.N % (p.y_dtype == DT_BF16 ? 8 : 4) == 0;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t nj = n0 + (wn * TN + j) * 32;
        if (nj >= p.N) break;
        Epi4 e[4] = {Epi4(p, nj + 4 * fhalf), Epi4(p, nj + 8 + 4 * fhalf), Epi4(p, nj + 16 + 4 * fhalf), Epi4(p, nj + 24 + 4 * fhalf)};
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int64_t mi = m0 + (wm * TM + i) * 32, m = mi + frow;
            const float sx = p.sx[m < p.M ? m : p.M - 1];
            if (p.y_dtype == DT_BF16 && whole) {
                // the halves of the wave swap what they hold of eight columns: a lane has sixteen, in two groups of 16 bytes
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x2 c[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int k = 2 * h + q;
                        const i32x4 sum = {acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]};
                        const f32x4 v = e[k](sum, sx);
                        c[q] = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                    }
                    u32x4 out;
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        const auto got = __builtin_amdgcn_permlane32_swap(c[0][d], c[1][d], false, false);
                        out[d] = got[0]; out[2 + d] = got[1];
                    }
                    const int64_t n = nj + 16 * h + 8 * fhalf;
                    if (m < p.M && n < p.N) *(u32x4 *)((uint16_t *)p.y + m * p.N + n) = out;
                }
                continue;
            }
            wave_lds_exchange();
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const i32x4 sum = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                *(f32x4 *)(park + frow * 32 + (((2 * q + fhalf) ^ (frow & 7)) << 2)) = e[q](sum, sx);
            }
            wave_lds_exchange();
            if (whole) {
#pragma unroll
                for (int h = 0; h < 4; ++h) {                       // 8 rows of 128 bytes
                    const int row = h * 8 + (lane >> 3), c = lane & 7;
                    const f32x4 a = *(const f32x4 *)(park + row * 32 + ((c ^ (row & 7)) << 2));
                    f32x4 *to = (f32x4 *)((float *)p.y + (mi + row) * p.N + nj + 4 * c);
                    if (mi + row < p.M && nj + 4 * c < p.N) {
                        // whole lines go past the L2, whose writing back the next operator would wait for: 4096 x 32000 x 1024 and the log probabilities
                        // behind it 134 -> 89 us for those, the product the same; lines in parts (of bf16, 8192 x 8192 x 4096) 270 -> 277
                        if (p.N % 32 == 0) {
                            asm volatile("");           // on both sides: else the two stores become one, an ordinary one
                            __builtin_nontemporal_store(a, to);
                            asm volatile("");
                        } else {
                            *to = a;
                        }
                    }
                }
            } else {
#pragma unroll 4
                for (int h = 0; h < 16; ++h) {                      // two rows, an element a lane
                    const int row = h * 2 + fhalf, c = frow;
                    const float a = park[row * 32 + (((c >> 2) ^ (row & 7)) << 2) + (c & 3)];
                    if (mi + row < p.M && nj + c < p.N) store_from_f32(p.y, p.y_dtype, (mi + row) * p.N + nj + c, a);
                }
            }
        }
    }
#endif
}

namespace {

template <int MT, int NT> void go_direct(const DenseQ8Params &p, hipStream_t s)
{
    Q8Grid g{(int32_t)((p.M + 16 * MT - 1) / (16 * MT)), (int32_t)((p.N + 16 * NT - 1) / (16 * NT)), (int32_t)(p.ldw / 128)};
    hipLaunchKernelGGL((dense_q8_direct_kernel<MT, NT>), dim3((unsigned)((int64_t)g.nblk_m * g.nblk_n)), dim3(512), 0, s, p, g);
}

template <int WM, int WN, int TM, int TN> void go_tile(const DenseQ8Params &p, hipStream_t s)
{
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    Q8Grid g{(int32_t)((p.M + BM - 1) / BM), (int32_t)((p.N + BN - 1) / BN), (int32_t)(p.ldw / 128)};
    hipLaunchKernelGGL((dense_q8_tile_kernel<WM, WN, TM, TN>), dim3((unsigned)((int64_t)g.nblk_m * g.nblk_n)), dim3(64 * WM * WN), 0, s, p, g);
}

// Which tile, by an estimate of the time: us per 128-byte line of K of a workgroup that is alone on its CU, and per line and 256 workgroups
// where there are more (measured; 8 x 4096 x 4096 from the smallest to the largest tile 7, 7, 9, 10, 14, 26, 32, 52 us, 128 x 4096 x 4096 32, 26,
// 19, 16, 20, 26, 33, 54, 2048 x 4096 x 4096 455, 353, 228, 196, 136, 65, 42, 58).  A tile's time beside its lines is not in it; for short rows it
// takes the fastest or one that is a little slower (4096 x 2048 x 1024 119, 109, 69, 66, 48, 20, 16.6, 22 us, of which it takes the seventh, 4096 x 1024 x 1024 60, 56, 36,
// 34, 25, 11.5, 11.9, 19, the seventh, 4096 x 8192 x 512 301, 302, 189, 175, 126, 52, 40, 38, the eighth, 512 x 2048 x 1024 18, 16, 11, 10, 8, 7, 11, 18, the fifth)
constexpr struct { int32_t bm, bn, threads; float alone, share; } forms[] = {
    {16, 16, 512, 0.14f, 0.14f}, {32, 16, 512, 0.16f, 0.19f}, {32, 32, 512, 0.23f, 0.25f}, {64, 32, 512, 0.41f, 0.40f}, {64, 64, 512, 0.55f, 0.55f},
    {64, 64, 256, 0.70f, 0.25f}, {128, 128, 256, 0.95f, 0.62f}, {256, 256, 512, 1.60f, 2.10f}};
int form_of(const DenseQ8Params &p)
{
    int best = 0;
    float least = INFINITY;
    for (int f = 0; f < 8; ++f) {
        const float wgs = (float)((p.M + forms[f].bm - 1) / forms[f].bm) * (float)((p.N + forms[f].bn - 1) / forms[f].bn);
        const float line = fmaxf(forms[f].alone, forms[f].share * wgs / 256.0f);
        if (line < least) { least = line; best = f; }
    }
    return best;
}

}  // namespace

bool dense_q8_fits(const DenseQ8Params &p)
{
    if (p.M < 1 || p.N < 1 || p.M > 0x7fffffff || p.N > 0x7fffffff) return false;
    const auto &f = forms[form_of(p)];
    return launch_has(((p.M + f.bm - 1) / f.bm) * ((p.N + f.bn - 1) / f.bn), f.threads);
}

hipError_t launch_dense_q8(const DenseQ8Params &p, hipStream_t s)
{
    if (p.M < 1 || p.N < 1 || p.K < 1 || p.K > 131071 || p.ldx < p.K || p.ldw < p.K || p.ldx % 16 != 0 || p.ldw % 128 != 0 || p.ldx > 131072 || p.ldw > 131072)
        return hipErrorInvalidValue;
    switch (form_of(p)) {
    case 0: go_direct<1, 1>(p, s); break;
    case 1: go_direct<2, 1>(p, s); break;
    case 2: go_direct<2, 2>(p, s); break;
    case 3: go_direct<4, 2>(p, s); break;
    case 4: go_direct<4, 4>(p, s); break;
    case 5: go_tile<2, 2, 1, 1>(p, s); break;
    case 6: go_tile<2, 2, 2, 2>(p, s); break;
    default: go_tile<2, 4, 4, 2>(p, s); break;
    }
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

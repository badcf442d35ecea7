// Gated linear recurrence over the rows of a sequence, every channel by itself:
//
//   h_t = a_t h_(t-1) + (1 - a_t) v_t,   a_t = sigmoid(f_t),   state in f32
//
// and its gradient, the same recurrence backwards: G_t = dh_t + a_(t+1) G_(t+1),
//   dv_t = G_t (1 - a_t),   df_t = G_t (h_(t-1) - v_t) a_t (1 - a_t).
// keep[t] = 0: padding, which holds the state; 2: the state before it is zero.
//
// A run of rows takes the state before it to A h + H, with A the product of its gates and H its own result from zero, and two runs
// one behind the other join as (A2 A1, A2 H1 + H2).  So a tile of 32 W runs of ROWS rows is worked off at once: a workgroup of W waves
// owns 32 lanes x 4 bytes of channels (whole 128-byte lines) and each half of a wave one run, which it reads once, into registers:
// prefix products and results of its rows from zero.  A run with a document's first row has -0 for A, which no product of gates
// is: nothing of what comes before goes into what follows, neither an infinity nor NaN.  The runs' (A, H) meet in LDS, every run adds up those before it, and one fma a
// row then gives the states.  The workgroup carries the tile's last state on to its next tile, whose rows are requested as
// the registers of this one's become free.  Nothing is read twice.  What bounds it is HBM, in columns of 128 bytes: 8 x 4096 x 2048 bf16 94 us
// (4.3 TB/s), its gradient 150 us (4.5 TB/s), both in turn 241; two tiles under way are no faster.  Fewer than 256 workgroups leave CUs without work: 8 x 1024 x
// 1024 is 128 of them, 18 and 26 us (2.8 and 3.3 TB/s).
//
// Few channels and many rows: each tile is a workgroup of its own.  A launch ahead finds the tiles' (A, H) (and, of the gradient, G),
// and every workgroup adds up those before (behind) its tile, at the cost of a second read: one sequence of 16384 x 1024 bf16 15 and 25 us.  The adding up
// grows with the square of the tiles: 131072 x 1024 in 345 us, where eight times the shorter sequence's 38 are 307.
#include <type_traits>

#include "igemm_lds.h"

namespace rl {

namespace {

// Rows of a run: as many as fit the registers with what they become, of two waves a SIMD where a workgroup walks its tiles, of four where
// tiles are workgroups (of the gradient, 8 x 4096 x 2048 bf16, forward and backward pass: 238 us with sixteen; 257 with eight and the rows of
// two tiles under way)
constexpr int FWD_ROWS = 16;
constexpr int bwd_rows(bool walks, bool keep) { return walks && !keep ? 16 : 8; }

// sigmoid(f) and 1 - sigmoid(f), each to its own last bits.  Below -87 the gate stays at e^-87, near the least f32 holds to all its bits: it
// leaves 6 of the largest state at most.
__device__ __forceinline__ void gate(float f, float &a, float &rest)
{
    const float e = __expf(-(f < -87.0f ? -87.0f : f));      // NaN stays NaN
    a = rcp_(1.0f + e);
    rest = e * a;
}

// 4 bytes (two bf16, one f32) or one bf16 of a row
template <typename E, int VEC> struct Raw { typedef uint32_t type; };
template <> struct Raw<uint16_t, 1> { typedef uint16_t type; };

template <typename E, int VEC> __device__ __forceinline__ float unpack(typename Raw<E, VEC>::type r, int j)
{
    if constexpr (sizeof(E) == 4) return __uint_as_float(r);
    else return j == 0 ? __uint_as_float((uint32_t)r << 16) : __uint_as_float((uint32_t)r & 0xffff0000u);
}

template <typename E, int VEC> __device__ __forceinline__ typename Raw<E, VEC>::type pack(const float (&v)[VEC])
{
    if constexpr (sizeof(E) == 4) return __float_as_uint(v[0]);
    else return (typename Raw<E, VEC>::type)pack_bf16x2(v[0], v[VEC - 1]);
}

// A x + H and A b of runs' A (KEEP: there may be documents' first rows)
constexpr float FIRST = -0.0f;
__device__ __forceinline__ bool is_first(float A) { return __float_as_uint(A) == 0x80000000u; }
template <bool KEEP> __device__ __forceinline__ float through(float A, float x, float H)
{
    const float y = __builtin_fmaf(A, x, H);
    return KEEP && is_first(A) ? H : y;
}
template <bool KEEP> __device__ __forceinline__ float both(float A, float b) { return KEEP && (is_first(A) || is_first(b)) ? FIRST : A * b; }
// A product of gates as it is used: at least the least number of f32, not 0, which no product of gates is.  An infinite state outlasts it and
// does not become NaN; a finite one is off by that number's share of it, a step of the last number there is.  As whole numbers, so that
// NaN stays and FIRST too.  The products themselves go on without it: it would be one more instruction a row that the next row waits for.
__device__ __forceinline__ float above_zero(float A) { return __uint_as_float(max(__float_as_uint(A), 1u)); }

// Rows of a tile in memory: `room` bytes from the tile's first row to the sequence's last.  What lies behind them reads as zero and is
// not written; so does what a lane without channels (offset OOB) asks for.
struct Rows { rsrc_t rsrc; };
__device__ __forceinline__ Rows rows_at(const void *first, int64_t room)
{
    return {make_rsrc(first, (uint32_t)(room < 0x7fffffff ? room : 0x7fffffff))};
}
template <typename R> __device__ __forceinline__ R load(const Rows &r, uint32_t off)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(R) == 4) return __builtin_amdgcn_raw_buffer_load_b32(r.rsrc, off, 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b16(r.rsrc, off, 0, 0);
#else
    return 0;
#endif
}
// STREAM: not kept in the L2, for results whose 128-byte lines each are one workgroup's (8 x 4096 x 2048 bf16 forward and backward pass: 247 ->
// 238 us; lines of two workgroups, 5 x 777 x 515 f32: 38.6 -> 42.2)
template <bool STREAM, typename R> __device__ __forceinline__ void store(const Rows &r, uint32_t off, R v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(R) == 4) __builtin_amdgcn_raw_buffer_store_b32(v, r.rsrc, off, 0, STREAM ? 2 : 0);
    else __builtin_amdgcn_raw_buffer_store_b16(v, r.rsrc, off, 0, STREAM ? 2 : 0);
#endif
}
// a value the compiler takes as new: what is made of it (the offsets of a tile's rows, unpacked operands) is made where it is used, not kept
// in registers from an earlier use
template <typename R> __device__ __forceinline__ R anew(R v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// What a lane works on: its channels of sequence b and its run of the tile's rows
template <typename E, int VEC, int ROWS, int W>
struct Place {
    static constexpr int TILE = 2 * W * ROWS;
    int wave, half, run;
    int32_t b, d, seg;                           // seg: blockIdx's tile where tiles are workgroups
    bool live;                                   // the channels exist
    uint32_t off1, off2;                         // bytes from a tile's first row to the run's, in rows of D and of 2 D
    __device__ __forceinline__ Place(const ScanParams &p, int32_t slabs)
    {
        const int lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        half = lane >> 5;
        run = 2 * wave + half;
        // where neighbours share lines they go to one XCD, whose L2 reads those once and writes them whole (both passes, 5 x 777 x 515 f32 packed 38.5 ->
        // 27.2 us, 8 x 1500 x 1000 f32 109 -> 84); with lines of their own one sequence of 16384 x 1024 bf16 is faster over all of them, 37.9 us not 40.5
        const uint32_t bid = p.D * sizeof(E) % 128 ? (uint32_t)xcd_run(blockIdx.x, gridDim.x) : blockIdx.x, rest = bid / (uint32_t)slabs, B = (uint32_t)p.B;
        seg = (int32_t)(rest / B);
        b = (int32_t)(rest - seg * B);
        d = (int32_t)((bid - rest * slabs) * 32 + (lane & 31)) * VEC;
        live = d < p.D;
        if (!live) d = 0;                        // its state is some other channel's, and nothing of it is stored
        off1 = live ? (uint32_t)((run * ROWS * (uint32_t)p.D + d) * sizeof(E)) : OOB;
        off2 = live ? (uint32_t)((run * ROWS * 2 * (uint32_t)p.D + d) * sizeof(E)) : OOB;
    }
};

// c, taken through tiles from .. to - 1 (BACK: to - 1 .. from) of `part`, whose vectors of a tile are `stride` floats apart, A first and
// the addend at `add`.  Every run of the workgroup joins its share of the tiles, then all of them the shares.
template <int VEC, int W, bool BACK, bool KEEP>
__device__ __forceinline__ void through_tiles(const float *part, int64_t stride, int64_t add, int32_t from, int32_t to, int run, float (&c)[VEC],
                                              float (&sa)[2 * W][32][VEC], float (&sx)[2 * W][32][VEC])
{
    const int n = to - from, l32 = threadIdx.x & 31;
    const int share = BACK ? 2 * W - 1 - run : run;
    const int32_t lo = from + (int32_t)((int64_t)n * share / (2 * W)), hi = from + (int32_t)((int64_t)n * (share + 1) / (2 * W));
    float a[VEC], x[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) { a[j] = 1.0f; x[j] = 0.0f; }
#pragma unroll 4
    for (int32_t k = lo; k < hi; ++k) {
        const float *q = part + (BACK ? lo + hi - 1 - k : k) * stride;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float ka = q[j];
            x[j] = through<KEEP>(ka, x[j], q[add + j]);
            a[j] = both<KEEP>(a[j], ka);
        }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) { sa[run][l32][j] = above_zero(a[j]); sx[run][l32][j] = x[j]; }
    __syncthreads();
#pragma unroll 4
    for (int r = 0; r < 2 * W; ++r)
#pragma unroll
        for (int j = 0; j < VEC; ++j) c[j] = through<KEEP>(sa[r][l32][j], c[j], sx[r][l32][j]);
}

// bit i: row t0 + i is padding (or past the sequence), is a document's first, is at or behind one of the run
template <int ROWS> struct Flags { uint32_t pad, first, behind; };
template <int ROWS, bool KEEP>
__device__ __forceinline__ Flags<ROWS> flags_of(const ScanParams &p, int64_t b, int64_t t0, int half)
{
    const int i = threadIdx.x & 31;
    const bool in = i < ROWS && t0 + i < p.T;
    const int k = !in ? 0 : KEEP ? p.keep[b * p.T + t0 + i] : 1;
    const uint64_t pad = __ballot(k == 0), first = __ballot(k == 2);
    const uint32_t f = (uint32_t)(first >> (32 * half));
    return {(uint32_t)(pad >> (32 * half)), f, (uint32_t)-(int32_t)(f & (uint32_t)-(int32_t)f)};
}

}  // namespace

// ---------------------------------------------------------------------------
// one token a sequence
// ---------------------------------------------------------------------------
template <typename E, int VEC>
__global__ __launch_bounds__(256) void linear_scan_step_kernel(const ScanParams p, int64_t total)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const int64_t c = i * VEC, b = c / p.D, d = c - b * p.D;
    typedef typename Raw<E, VEC>::type raw_t;
    const raw_t f = *(const raw_t *)((const E *)p.z + 2 * b * p.D + d), v = *(const raw_t *)((const E *)p.z + (2 * b + 1) * p.D + d);
    const int keep = p.keep ? p.keep[b] : 1;
    float out[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        float a, rest, h = p.h0[c + j];
        gate(unpack<E, VEC>(f, j), a, rest);
        const float u = rest * unpack<E, VEC>(v, j);
        if (keep) h = keep == 2 ? u : __builtin_fmaf(a, h, u);
        p.hT[c + j] = h;
        out[j] = keep ? h : 0.0f;
    }
    *(raw_t *)((E *)p.h + c) = pack<E, VEC>(out);
}

// ---------------------------------------------------------------------------
// forward.  MODE 0: a workgroup walks its channels' tiles; 1: (A, H) of one tile into part; 2: one tile, after those before it
// ---------------------------------------------------------------------------
template <typename E, int VEC, int W, int MODE, bool KEEP, bool STREAM>
__global__ __launch_bounds__(64 * W, MODE == 0 ? 2 : 4) void linear_scan_kernel(const ScanParams p, int32_t slabs, int32_t tiles)
{
    constexpr int ROWS = FWD_ROWS, AT_ONCE = MODE == 0 ? W : 4;      // other waves' sums read at once: those of all where there are registers for them
    typedef Place<E, VEC, ROWS, W> P;
    typedef typename Raw<E, VEC>::type raw_t;
    const P at(p, slabs);
    const int64_t BD = p.B * p.D, chan = at.b * p.D + at.d;
    const uint32_t line = (uint32_t)p.D * sizeof(E);
    __shared__ float sa[2][W][32][VEC], sh[2][W][32][VEC];
    const int l32 = threadIdx.x & 31;

    raw_t rf[ROWS], rv[ROWS];
    auto rows_of = [&](const void *x, int64_t tile, int wide) {              // rows of `wide` lines
        const int64_t t = tile * P::TILE;
        return rows_at((const char *)x + (at.b * p.T + t) * wide * line, (p.T - t) * wide * line);
    };
    const int32_t first_tile = MODE ? at.seg : 0, last_tile = MODE ? at.seg + 1 : tiles;
    Rows z = rows_of(p.z, first_tile, 2);
    auto request = [&](uint32_t off, int i) {
        rf[i] = load<raw_t>(z, off + 2 * i * line);
        rv[i] = load<raw_t>(z, off + (2 * i + 1) * line);
    };
#pragma unroll
    for (int i = 0; i < ROWS; ++i) request(at.off2, i);

    float carry[VEC];
    if (MODE != 1) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) carry[j] = p.h0[chan + j];
        if constexpr (MODE == 2) {
            __shared__ float ta[2 * W][32][VEC], th[2 * W][32][VEC];
            through_tiles<VEC, W, false, KEEP>(p.part + chan, 2 * BD, BD, 0, at.seg, at.run, carry, ta, th);
        }
    }
    for (int32_t tile = first_tile; tile < last_tile; ++tile) {
        const int64_t t0 = (int64_t)tile * P::TILE + at.run * ROWS;
        const bool whole = (int64_t)(tile + 1) * P::TILE <= p.T;
        const uint32_t off2 = anew(at.off2), off1 = anew(at.off1);
        if (MODE == 0 && tile + 1 < last_tile) z = rows_of(p.z, tile + 1, 2);
        float A[ROWS][VEC], H[ROWS][VEC];
        Flags<ROWS> fl{0, 0, 0};
        float pa[VEC], ph[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) { pa[j] = 1.0f; ph[j] = 0.0f; }
        auto rows = [&](auto masked) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const raw_t qf = MODE == 0 ? rf[i] : anew(rf[i]), qv = MODE == 0 ? rv[i] : anew(rv[i]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float a, rest;
                    gate(unpack<E, VEC>(qf, j), a, rest);
                    float u = rest * unpack<E, VEC>(qv, j);
                    if (masked) {
                        const bool pad = fl.pad >> i & 1u;
                        a = pad ? 1.0f : a;
                        u = pad ? 0.0f : u;
                        if (KEEP && (fl.first >> i & 1u)) ph[j] = 0.0f;
                    }
                    pa[j] *= a;
                    ph[j] = __builtin_fmaf(a, ph[j], u);
                    A[i][j] = above_zero(pa[j]); H[i][j] = ph[j];
                }
                if (MODE == 0 && tile + 1 < last_tile) request(off2, i);
            }
        };
        if (KEEP || !whole) fl = flags_of<ROWS, KEEP>(p, at.b, t0, at.half);
        // with a keep every row is masked: a second loop for waves of tokens alone is slower (8 x 4096 x 2048 bf16, documents of some 400 tokens,
        // forward pass 93 -> 96 us, both passes 241 -> 249): what bounds either is memory
        const bool masked = KEEP || !whole;
        if (masked) rows(std::true_type{});
        else rows(std::false_type{});
#pragma unroll
        for (int j = 0; j < VEC; ++j) pa[j] = KEEP && fl.first != 0 ? FIRST : above_zero(pa[j]);
        // the wave's two runs as one, the waves' in LDS
        float oa[VEC], oh[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) { oa[j] = __shfl_xor(pa[j], 32); oh[j] = __shfl_xor(ph[j], 32); }
        const int buf = MODE == 0 ? tile & 1 : 0;
        if (at.half) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                sa[buf][at.wave][l32][j] = above_zero(both<KEEP>(pa[j], oa[j]));
                sh[buf][at.wave][l32][j] = through<KEEP>(pa[j], oh[j], ph[j]);
            }
        }
        if (W > 1) __syncthreads(); else wave_lds_exchange();
        float mine[VEC];
        if (MODE == 1) {
            if (at.run == 0 && at.live) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float ta = 1.0f, th = 0.0f;
#pragma unroll
                    for (int w = 0; w < W; ++w) { th = through<KEEP>(sa[0][w][l32][j], th, sh[0][w][l32][j]); ta = both<KEEP>(ta, sa[0][w][l32][j]); }
                    p.part[2 * at.seg * BD + chan + j] = above_zero(ta);
                    p.part[(2 * at.seg + 1) * BD + chan + j] = th;
                }
            }
            return;
        }
#pragma unroll AT_ONCE
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (w == at.wave) mine[j] = carry[j];
                carry[j] = through<KEEP>(sa[buf][w][l32][j], carry[j], sh[buf][w][l32][j]);
            }
        if (at.half) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) mine[j] = through<KEEP>(oa[j], mine[j], oh[j]);
        }
        if (at.live) {
            if (p.states && t0 % p.state_rows == 0 && t0 < p.T) {
                const int64_t count = (p.T + p.state_rows - 1) / p.state_rows;
#pragma unroll
                for (int j = 0; j < VEC; ++j) p.states[(at.b * count + t0 / p.state_rows) * p.D + at.d + j] = mine[j];
            }
            if (p.h) {
                const Rows h = rows_of(p.h, tile, 1);
                auto results = [&](auto masked) {
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        float out[VEC];
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            out[j] = masked && (fl.behind >> i & 1u) ? H[i][j] : __builtin_fmaf(A[i][j], mine[j], H[i][j]);
                            if (masked && (fl.pad >> i & 1u)) out[j] = 0.0f;
                        }
                        store<STREAM>(h, off1 + i * line, pack<E, VEC>(out));
                    }
                };
                results(std::bool_constant<KEEP>{});
            }
            if (p.hT && tile + 1 == tiles && at.run == 0) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) p.hT[chan + j] = carry[j];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// gradient.  MODE as above, tiles from the last to the first; part: A, H, G of a tile.  The state before a tile comes from p.states
// (MODE 0) or from the tiles before it (MODE 2).
// ---------------------------------------------------------------------------
template <typename E, int VEC, int W, int MODE, bool KEEP, bool STREAM>
__global__ __launch_bounds__(64 * W, MODE == 0 ? 2 : 4) void linear_scan_grad_kernel(const ScanParams p, int32_t slabs, int32_t tiles)
{
    constexpr int ROWS = bwd_rows(MODE == 0, KEEP), AT_ONCE = MODE == 0 ? W : 4;
    typedef Place<E, VEC, ROWS, W> P;
    typedef typename Raw<E, VEC>::type raw_t;
    const P at(p, slabs);
    const int64_t BD = p.B * p.D, chan = at.b * p.D + at.d;
    const uint32_t line = (uint32_t)p.D * sizeof(E);
    __shared__ float sa[2][W][32][VEC], sh[2][W][32][VEC], sg[2][W][32][VEC];
    const int l32 = threadIdx.x & 31;

    raw_t rf[ROWS], rv[ROWS], rd[ROWS];
    auto rows_of = [&](const void *x, int64_t tile, int wide) {              // rows of `wide` lines
        const int64_t t = tile * P::TILE;
        return rows_at((const char *)x + (at.b * p.T + t) * wide * line, (p.T - t) * wide * line);
    };
    const int32_t first_tile = MODE ? at.seg : tiles - 1, last_tile = MODE ? at.seg - 1 : -1;
    Rows z = rows_of(p.z, first_tile, 2), d = rows_of(p.dh, first_tile, 1);
    auto request = [&](uint32_t off2, uint32_t off1, int i) {
        rf[i] = load<raw_t>(z, off2 + 2 * i * line);
        rv[i] = load<raw_t>(z, off2 + (2 * i + 1) * line);
        rd[i] = load<raw_t>(d, off1 + i * line);
    };
#pragma unroll
    for (int i = 0; i < ROWS; ++i) request(at.off2, at.off1, i);

    const int64_t count = p.states ? (p.T + p.state_rows - 1) / p.state_rows : 0;
    float gcarry[VEC], start[VEC];
    if (MODE != 1) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) gcarry[j] = p.dhT[chan + j];
        if constexpr (MODE == 2) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) start[j] = p.h0[chan + j];
            __shared__ float ta[2][2 * W][32][VEC], tx[2][2 * W][32][VEC];
            through_tiles<VEC, W, false, KEEP>(p.part + chan, 3 * BD, BD, 0, at.seg, at.run, start, ta[0], tx[0]);
            through_tiles<VEC, W, true, KEEP>(p.part + chan, 3 * BD, 2 * BD, at.seg + 1, tiles, at.run, gcarry, ta[1], tx[1]);
        }
    }
    for (int32_t tile = first_tile; tile > last_tile; --tile) {
        const int64_t t0 = (int64_t)tile * P::TILE + at.run * ROWS;
        const bool whole = (int64_t)(tile + 1) * P::TILE <= p.T;
        const uint32_t off2 = anew(at.off2), off1 = anew(at.off1);
        if (MODE == 0 && tile > 0) { z = rows_of(p.z, tile - 1, 2); d = rows_of(p.dh, tile - 1, 1); }
        if (MODE == 0) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) start[j] = tile ? p.states[(at.b * count + tile) * p.D + at.d + j] : p.h0[chan + j];
        }
        float a[ROWS][VEC], rest[ROWS][VEC], before[ROWS][VEC];   // before: of the state before the row, the run's own part
        raw_t kv[ROWS], kd[ROWS];
        float pa[VEC], ph[VEC], pg[VEC];
        Flags<ROWS> fl{0, 0, 0};
#pragma unroll
        for (int j = 0; j < VEC; ++j) { pa[j] = 1.0f; ph[j] = 0.0f; pg[j] = 0.0f; }
        auto rows = [&](auto masked) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    gate(unpack<E, VEC>(rf[i], j), a[i][j], rest[i][j]);
                    float u = rest[i][j] * unpack<E, VEC>(rv[i], j);
                    float af = a[i][j], dh = unpack<E, VEC>(rd[i], j);
                    if (masked) {
                        const bool pad = fl.pad >> i & 1u;
                        dh = pad ? 0.0f : dh;
                        af = pad ? 1.0f : af;
                        u = pad ? 0.0f : u;
                        if (KEEP && (fl.first >> i & 1u)) ph[j] = 0.0f;
                    }
                    const bool behind = KEEP && masked && (fl.behind >> i & 1u);
                    before[i][j] = ph[j];
                    pa[j] *= af;
                    ph[j] = __builtin_fmaf(af, ph[j], u);
                    if (!behind) pg[j] = __builtin_fmaf(above_zero(pa[j]), dh, pg[j]);
                }
                kv[i] = rv[i]; kd[i] = rd[i];
                if (MODE == 0 && tile > 0) request(off2, off1, i);
            }
        };
        if (KEEP || !whole) fl = flags_of<ROWS, KEEP>(p, at.b, t0, at.half);
        const bool masked = KEEP || !whole;
        if (masked) rows(std::true_type{});
        else rows(std::false_type{});
        // the rows' masks are made again for the way back: kept from here they are more scalar registers than there are (both passes 246 -> 235 us)
        if (KEEP && MODE == 0) fl = {anew(fl.pad), anew(fl.first), anew(fl.behind)};
#pragma unroll
        for (int j = 0; j < VEC; ++j) pa[j] = KEEP && fl.first != 0 ? FIRST : above_zero(pa[j]);
        float oa[VEC], oh[VEC], og[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) { oa[j] = __shfl_xor(pa[j], 32); oh[j] = __shfl_xor(ph[j], 32); og[j] = __shfl_xor(pg[j], 32); }
        const int buf = MODE == 0 ? tile & 1 : 0;
        if (at.half) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                sa[buf][at.wave][l32][j] = above_zero(both<KEEP>(pa[j], oa[j]));
                sh[buf][at.wave][l32][j] = through<KEEP>(pa[j], oh[j], ph[j]);
                sg[buf][at.wave][l32][j] = through<KEEP>(oa[j], pg[j], og[j]);
            }
        }
        if (W > 1) __syncthreads(); else wave_lds_exchange();
        if (MODE == 1) {
            if (at.run == 0 && at.live) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float ta = 1.0f, th = 0.0f, tg = 0.0f;
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        tg = through<KEEP>(above_zero(ta), sg[0][w][l32][j], tg);
                        th = through<KEEP>(sa[0][w][l32][j], th, sh[0][w][l32][j]);
                        ta = both<KEEP>(ta, sa[0][w][l32][j]);
                    }
                    p.part[3 * at.seg * BD + chan + j] = above_zero(ta);
                    p.part[(3 * at.seg + 1) * BD + chan + j] = th;
                    p.part[(3 * at.seg + 2) * BD + chan + j] = tg;
                }
            }
            return;
        }
        float h[VEC], G[VEC], c[VEC];
        // the states and gradients that reach the wave, the gradient on to the next tile
#pragma unroll
        for (int j = 0; j < VEC; ++j) c[j] = start[j];
#pragma unroll AT_ONCE
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (w == at.wave) h[j] = c[j];
                c[j] = through<KEEP>(sa[buf][w][l32][j], c[j], sh[buf][w][l32][j]);
            }
#pragma unroll AT_ONCE
        for (int w = W - 1; w >= 0; --w)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (w == at.wave) G[j] = gcarry[j];
                gcarry[j] = through<KEEP>(sa[buf][w][l32][j], gcarry[j], sg[buf][w][l32][j]);
            }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (at.half) h[j] = through<KEEP>(oa[j], h[j], oh[j]);
            else G[j] = through<KEEP>(oa[j], G[j], og[j]);
        }
        if (at.live) {
            // the state before every row, then the rows backwards
            auto replay = [&](auto masked) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float run = h[j];                        // the start times the gates so far
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        if (KEEP && masked && (fl.first >> i & 1u)) run = 0.0f;
                        before[i][j] += run;
                        run *= masked && (fl.pad >> i & 1u) ? 1.0f : a[i][j];
                    }
                }
                const Rows dz = rows_of(p.dz, tile, 2);
#pragma unroll
                for (int i = ROWS - 1; i >= 0; --i) {
                    const raw_t qv = MODE == 0 ? kv[i] : anew(kv[i]), qd = MODE == 0 ? kd[i] : anew(kd[i]);
                    float df[VEC], dv[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float g = G[j] + unpack<E, VEC>(qd, j);
                        dv[j] = g * rest[i][j];
                        df[j] = dv[j] * (before[i][j] - unpack<E, VEC>(qv, j)) * a[i][j];
                        const float on = a[i][j] * g;
                        if (masked) {
                            const bool pad = fl.pad >> i & 1u;
                            G[j] = pad ? G[j] : fl.first >> i & 1u ? 0.0f : on;
                            dv[j] = pad ? 0.0f : dv[j];
                            df[j] = pad ? 0.0f : df[j];
                        } else {
                            G[j] = on;
                        }
                    }
                    store<STREAM>(dz, off2 + 2 * i * line, pack<E, VEC>(df));
                    store<STREAM>(dz, off2 + (2 * i + 1) * line, pack<E, VEC>(dv));
                }
            };
            if (masked) replay(std::true_type{});
            else replay(std::false_type{});
            if (tile == 0 && at.run == 0) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) p.dh0[chan + j] = gcarry[j];
            }
        }
    }
}

// ---------------------------------------------------------------------------
namespace {

struct Form { int W, rows; bool split; int32_t slabs, tiles; };

// channels of a lane
int lane_channels(const ScanParams &p) { return p.dtype == DT_BF16 && p.D % 2 == 0 ? 2 : 1; }

// Waves of a workgroup: enough for the rows, eight where there are few workgroups.  split: tiles as workgroups of their own, where there are
// fewer than 128 workgroups that walk (channels of 64 x rows, bf16, forward pass: 64 x 2400 walking 33 us, split 23; 128 x 2400 39 and 42;
// 192 x 2400 44 and 62; both passes 16 x 600 27 and 18, 128 x 2400 106 and 107); of four waves up to some 4000 rows, eight from there on
// (both passes, 64 x 2400 58 and 62 us, 16 x 16384 112 and 102)
Form form_of(const ScanParams &p, bool grad)
{
    const int64_t vec = lane_channels(p);
    Form f;
    f.slabs = (int32_t)((p.D + 32 * vec - 1) / (32 * vec));
    const int64_t wgs = p.B * f.slabs;
    f.split = false;
    for (int walks = 1; walks >= 0; --walks) {
        f.rows = grad ? bwd_rows(walks, p.keeps) : FWD_ROWS;
        f.W = p.T <= 2 * f.rows ? 1 : p.T <= 8 * f.rows || wgs >= 512 || (!walks && p.T < 4096) ? 4 : 8;
        f.tiles = (int32_t)((p.T + 2 * f.W * f.rows - 1) / (2 * f.W * f.rows));
        if (wgs >= 128 || f.tiles == 1) break;
        f.split = true;
    }
    return f;
}

template <typename E, int VEC, int W, int MODE, bool STREAM>
void go(bool grad, const ScanParams &p, const Form &f, hipStream_t s)
{
    const dim3 grid((unsigned)(p.B * f.slabs * (MODE ? f.tiles : 1))), wg(64 * W);
    if (grad) {
        if (p.keep) hipLaunchKernelGGL((linear_scan_grad_kernel<E, VEC, W, MODE, true, STREAM>), grid, wg, 0, s, p, f.slabs, f.tiles);
        else hipLaunchKernelGGL((linear_scan_grad_kernel<E, VEC, W, MODE, false, STREAM>), grid, wg, 0, s, p, f.slabs, f.tiles);
    } else {
        if (p.keep) hipLaunchKernelGGL((linear_scan_kernel<E, VEC, W, MODE, true, STREAM>), grid, wg, 0, s, p, f.slabs, f.tiles);
        else hipLaunchKernelGGL((linear_scan_kernel<E, VEC, W, MODE, false, STREAM>), grid, wg, 0, s, p, f.slabs, f.tiles);
    }
}

template <typename E, int VEC, int W, int MODE>
void go(bool grad, const ScanParams &p, const Form &f, hipStream_t s)
{
    if constexpr (MODE != 1 && VEC * sizeof(E) == 4) {             // the others store nothing, have no whole lines
        if (p.D * sizeof(E) % 128 == 0) return go<E, VEC, W, MODE, true>(grad, p, f, s);
    }
    go<E, VEC, W, MODE, false>(grad, p, f, s);
}

template <typename E, int VEC>
void go(bool grad, int mode, const ScanParams &p, const Form &f, hipStream_t s)
{
    if (mode == 1) f.W == 4 ? go<E, VEC, 4, 1>(grad, p, f, s) : go<E, VEC, 8, 1>(grad, p, f, s);
    else if (mode == 2) f.W == 4 ? go<E, VEC, 4, 2>(grad, p, f, s) : go<E, VEC, 8, 2>(grad, p, f, s);
    else if (f.W == 1) go<E, VEC, 1, 0>(grad, p, f, s);
    else if (f.W == 4) go<E, VEC, 4, 0>(grad, p, f, s);
    else go<E, VEC, 8, 0>(grad, p, f, s);
}

void go(bool grad, int mode, const ScanParams &p, const Form &f, hipStream_t s)
{
    if (p.dtype != DT_BF16) go<float, 1>(grad, mode, p, f, s);
    else if (p.D % 2 == 0) go<uint16_t, 2>(grad, mode, p, f, s);
    else go<uint16_t, 1>(grad, mode, p, f, s);
}

bool sizes_ok(const ScanParams &p)
{
    // a tile's rows are reached by 31-bit offsets
    return p.B >= 1 && p.T >= 1 && p.D >= 1 && p.B <= 0x7fffffff && p.T <= 0x7fffffff && p.D <= SCAN_MAX_D;
}

}  // namespace

bool scan_fits(const ScanParams &p, bool grad)
{
    if (!sizes_ok(p)) return false;
    if (p.T == 1 && !grad) return launch_has((p.B * p.D / lane_channels(p) + 255) / 256, 256);
    const Form f = form_of(p, grad);
    return launch_has(p.B * f.slabs * (f.split ? f.tiles : 1), 64 * f.W);
}

int64_t scan_state_rows(const ScanParams &p)
{
    const Form f = form_of(p, true);
    return f.split || f.tiles == 1 ? 0 : 2 * f.W * f.rows;
}

int64_t scan_part_floats(const ScanParams &p, bool grad)
{
    const Form f = form_of(p, grad);
    return f.split ? (grad ? 3 : 2) * f.tiles * p.B * p.D : 0;
}

hipError_t launch_scan(const ScanParams &p, hipStream_t s)
{
    const Form f = form_of(p, false);
    if (!sizes_ok(p) || p.keeps != (p.keep != nullptr) || (f.split && !p.part) || (p.states && p.state_rows % FWD_ROWS != 0)) return hipErrorInvalidValue;
    if (p.T == 1) {                                // (states alone are of longer sequences)
        if (!p.h || !p.hT) return hipErrorInvalidValue;
        const int vec = lane_channels(p);
        const int64_t total = p.B * p.D / vec, blocks = (total + 255) / 256;
        if (p.dtype != DT_BF16) hipLaunchKernelGGL((linear_scan_step_kernel<float, 1>), dim3((unsigned)blocks), dim3(256), 0, s, p, total);
        else if (vec == 2) hipLaunchKernelGGL((linear_scan_step_kernel<uint16_t, 2>), dim3((unsigned)blocks), dim3(256), 0, s, p, total);
        else hipLaunchKernelGGL((linear_scan_step_kernel<uint16_t, 1>), dim3((unsigned)blocks), dim3(256), 0, s, p, total);
        return hipGetLastError();
    }
    if (f.split) go(false, 1, p, f, s);
    go(false, f.split ? 2 : 0, p, f, s);
    return hipGetLastError();
}

hipError_t launch_scan_grad(const ScanParams &p, hipStream_t s)
{
    const Form f = form_of(p, true);
    if (!sizes_ok(p) || p.keeps != (p.keep != nullptr) || (f.split && !p.part) || (!f.split && f.tiles > 1 && (!p.states || p.state_rows != 2 * f.W * f.rows))) return hipErrorInvalidValue;
    if (f.split) go(true, 1, p, f, s);
    go(true, f.split ? 2 : 0, p, f, s);
    return hipGetLastError();
}

}  // namespace rl

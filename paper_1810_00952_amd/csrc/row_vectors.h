// A row of a matrix held by a workgroup as the 16-byte vectors of memory, whatever the row's alignment.
#pragma once
#include "igemm_lds.h"

namespace rl {

namespace {

// the same value as one of its own: what is made of it is not kept in registers from one use for the next
__device__ __forceinline__ u32x4 anew(u32x4 v)
{
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ int32_t anew(int32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// Sum and maximum over the wave, in every lane: rows of sixteen lanes by shifts, then the rows one into the next, without the LDS that a
// shuffle goes through (six dependent instructions, not six round trips).  All lanes have to be active.
template <bool MAX> __device__ __forceinline__ float over_wave(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
#define RL_STEP(CTRL, ROWS)                                                                                                        \
    {                                                                                                                              \
        const int o = __builtin_amdgcn_update_dpp(MAX ? __builtin_bit_cast(int, v) : 0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false); \
        v = MAX ? fmaxf(v, __builtin_bit_cast(float, o)) : v + __builtin_bit_cast(float, o);                                       \
    }
    RL_STEP(0x111, 0xf) RL_STEP(0x112, 0xf) RL_STEP(0x114, 0xf) RL_STEP(0x118, 0xf)      // row_shr 1, 2, 4, 8
    RL_STEP(0x142, 0xa) RL_STEP(0x143, 0xc)                                              // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
#undef RL_STEP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
#else
    return v;
#endif
}
__device__ __forceinline__ float wave_sum(float v) { return over_wave<false>(v); }
__device__ __forceinline__ float wave_max(float v) { return over_wave<true>(v); }

template <typename E> __device__ __forceinline__ float unpack(const u32x4 &r, int k)
{
    if constexpr (sizeof(E) == 4) return __uint_as_float(r[k]);
    else return __uint_as_float((k & 1) ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
}
template <typename E> __device__ __forceinline__ u32x4 pack(const float *v)
{
    u32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = sizeof(E) == 4 ? __float_as_uint(v[k]) : pack_bf16x2(v[2 * k], v[2 * k + 1]);
    return r;
}

// Columns lo .. hi - 1 of row r of a matrix of V columns of E (uint16_t: bf16).  Vector j of thread t covers columns
// first + N (j T + t) .. + N - 1, at a multiple of 16 bytes.  Of vector 0 and of the last only a part may lie in lo .. hi - 1: those are
// read and written an element at a time, by the thread that has them.
template <typename E, int T, int NV>
struct RowVectors {
    static constexpr int N = 16 / sizeof(E);
    int32_t lo, hi, first, used;                // used: vectors a thread has at most
    int32_t last_j, last_t;                     // whose the last vector is
    bool head, tail;                            // the first, the last vector is the thread's and cut

    __device__ __forceinline__ RowVectors(int64_t r, int64_t V, int32_t lo_, int32_t hi_) : lo(lo_), hi(hi_)
    {
        first = lo - (int32_t)((r * V + lo) % N);
        const int32_t last = (hi - 1 - first) / N;
        used = last / T + 1;
        last_j = last / T; last_t = last % T;
        head = threadIdx.x == 0 && first < lo;
        tail = (int32_t)threadIdx.x == last_t && first + (last + 1) * N > hi;
    }
    __device__ __forceinline__ int32_t column(int j) const { return first + N * (j * T + (int32_t)threadIdx.x); }
    // whether the thread's vector j is there and whole; false of the cut ones
    __device__ __forceinline__ bool whole(int j) const
    {
        return !(j == 0 && head) && (j < last_j || (int32_t)threadIdx.x < last_t || ((int32_t)threadIdx.x == last_t && !tail));
    }
    // bytes from vector j of thread 0, of elements of `size` bytes
    __device__ __forceinline__ uint32_t offset(int j, int size = sizeof(E)) const
    {
        return (j != 0 && j != last_j) || whole(j) ? threadIdx.x * (uint32_t)(N * size) : OOB;
    }
    __device__ __forceinline__ u32x4 cut(const E *row, int32_t c, uint32_t fill) const
    {
        u32x4 v = {fill, fill, fill, fill};
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (c + k >= lo && c + k < hi) {
                if constexpr (sizeof(E) == 4) v[k] = ((const uint32_t *)row)[c + k];
                else v[k >> 1] = (k & 1) ? (v[k >> 1] & 0xffffu) | (uint32_t)((const uint16_t *)row)[c + k] << 16
                                         : (v[k >> 1] & 0xffff0000u) | ((const uint16_t *)row)[c + k];
            }
        return v;
    }
    // row: its column 0.  What is no column of lo .. hi - 1 becomes `fill`; vectors from `used` on are left alone
    __device__ __forceinline__ void load(const E *row, uint32_t fill, u32x4 (&x)[NV]) const
    {
#if defined(__HIP_DEVICE_COMPILE__)
        const rsrc_t src = make_rsrc(row + first, 0x7fffffffu);
        const u32x4 nothing = {fill, fill, fill, fill};
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < used) x[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src, offset(j), j * T * 16, 0));
        if (!whole(0)) x[0] = nothing;
        if (head) x[0] = cut(row, first, fill);
        u32x4 end = nothing;
        if (tail) end = cut(row, column(last_j), fill);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j == last_j && !whole(j) && !(j == 0 && head)) x[j] = end;
#endif
    }
    // the thread's vectors of a result of the row's shape, one at a time, then finish
    // (past the L2: 16384 x 4096 bf16 norm with residual and a reader of its 8-bit values 253 -> 237 us, 2000 x 10007 f32 log probabilities with
    // their gradient 36.9 -> 31.3; of 8192 x 32000 bf16 the operator 199 -> 222 us and the gradient's first reader 490 -> 470: no more, no less)
    struct Out { rsrc_t dst; u32x4 first, last; };
    __device__ __forceinline__ Out out(E *row) const { return {make_rsrc(row + first, 0x7fffffffu), {}, {}}; }
    __device__ __forceinline__ void put(Out &o, int j, u32x4 v) const
    {
#if defined(__HIP_DEVICE_COMPILE__)
        __builtin_amdgcn_raw_buffer_store_b128(v, o.dst, offset(j), j * T * 16, 2);
        if (j == 0) o.first = v;
        if (j == last_j) o.last = v;
#endif
    }
    __device__ __forceinline__ void put_cut(E *row, int32_t c, const u32x4 &v) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (c + k >= lo && c + k < hi) {
                if constexpr (sizeof(E) == 4) ((uint32_t *)row)[c + k] = v[k];
                else row[c + k] = (E)(v[k >> 1] >> (16 * (k & 1)));
            }
    }
    __device__ __forceinline__ void finish(const Out &o, E *row) const
    {
        if (head) put_cut(row, first, o.first);
        if (tail && !(head && last_j == 0)) put_cut(row, column(last_j), o.last);
    }
    // the same of a result of one byte an element; v: N bytes
    struct OutBytes { rsrc_t dst; u32x2 first, last; };
    __device__ __forceinline__ OutBytes out_bytes(int8_t *row) const { return {make_rsrc(row + first, 0x7fffffffu), {}, {}}; }
    __device__ __forceinline__ void put(OutBytes &o, int j, u32x2 v) const
    {
#if defined(__HIP_DEVICE_COMPILE__)
        if constexpr (N == 8) __builtin_amdgcn_raw_buffer_store_b64(v, o.dst, offset(j, 1), j * T * N, 0);
        else __builtin_amdgcn_raw_buffer_store_b32(v[0], o.dst, offset(j, 1), j * T * N, 0);
        if (j == 0) o.first = v;
        if (j == last_j) o.last = v;
#endif
    }
    __device__ __forceinline__ void put_cut(int8_t *row, int32_t c, const u32x2 &v) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (c + k >= lo && c + k < hi) row[c + k] = (int8_t)(v[k >> 2] >> (8 * (k & 3)));
    }
    __device__ __forceinline__ void finish(const OutBytes &o, int8_t *row) const
    {
        if (head) put_cut(row, first, o.first);
        if (tail && !(head && last_j == 0)) put_cut(row, column(last_j), o.last);
    }
};

}  // namespace

}  // namespace rl

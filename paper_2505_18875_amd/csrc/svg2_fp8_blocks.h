// E4M3 operands with one power of two for each block of 128: what their kernels and the layer norm that writes such operands share
// (internal header).
//
// A block of 128 values along the contracted axis shares one power of two, kept as its exponent + 127 in a byte (255: NaN), the smallest for
// which max |x| <= 448 * 2^exponent, at least 2^-127: nothing saturates.  Storage of R rows and K columns, Kp = K rounded up to 128: codes
// [R, Kp], zeros behind K; scales [ceil(Kp / 512), R, 4], block b of row r at [b / 4, r, b % 4], zeros behind the last block.
#pragma once

#include "svg2_common.h"

namespace svg2 {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));     // 16 bytes at any element's address: one load or store all the same
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return bf16_to_f32(x); }

// two fp32 -> two bf16, to nearest even (NaN stays NaN)
__device__ __forceinline__ unsigned pack_bf16(float a, float b)
{
    const f32x2 p = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
}

__device__ __forceinline__ void store_one(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_one(bf16_t *p, float v) { *p = (bf16_t)pack_bf16(v, 0.f); }

// |x| as bits: they order like the magnitudes, NaN above infinity
__device__ __forceinline__ unsigned mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Eight neighbouring columns as they are in memory.
template <typename T> struct Raw { u32x4 q[sizeof(T) / 2]; };

// STREAM, here and below: past the caches
template <typename T, bool STREAM = false> __device__ __forceinline__ Raw<T> load_raw(const T *from)
{
    const u32x4_any *p = reinterpret_cast<const u32x4_any *>(from);
    Raw<T> r;
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) r.q[i] = STREAM ? __builtin_nontemporal_load(p + i) : p[i];
    return r;
}

// f(0) .. f(7)
template <typename T, typename F> __device__ __forceinline__ Raw<T> raw_of(F f)
{
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = f(i);
    Raw<T> r;
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (sizeof(T) == 4) r.q[i][w] = __float_as_uint(e[4 * i + w]);
            else r.q[i][w] = e[2 * w] | (unsigned)e[2 * w + 1] << 16;
        }
    return r;
}

// columns k .. k + 7 of a row, zeros behind D
template <typename T> __device__ __forceinline__ Raw<T> load_raw(const T *row, int k, int D)
{
    if (k + 8 <= D) return load_raw<T>(row + k);
    return raw_of<T>([&](int i) { return k + i < D ? row[k + i] : (T)0; });
}

// value i of the eight
template <typename T> __device__ __forceinline__ float value(const Raw<T> &r, int i)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(r.q[i >> 2][i & 3]);
    else return __uint_as_float(i & 1 ? r.q[0][i >> 1] & 0xFFFF0000u : r.q[0][i >> 1] << 16);
}

template <typename T> __device__ __forceinline__ void decode(const Raw<T> &r, float *v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value<T>(r, i);
}

// eight neighbouring elements from and to any address
template <typename T> __device__ __forceinline__ void load8(const T *from, float *v) { decode<T>(load_raw<T>(from), v); }

template <typename T, bool STREAM = false> __device__ __forceinline__ void store8(T *to, const float *v)
{
    u32x4_any *p = reinterpret_cast<u32x4_any *>(to);
    auto store = [](const u32x4 &x, u32x4_any *at) {
        if (STREAM) __builtin_nontemporal_store(x, at);
        else *at = x;
    };
    if constexpr (sizeof(T) == 4) {
        store(u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, p);
        store(u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}, p + 1);
    } else store(u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}, p);
}

// bits of the largest magnitude of eight values
__device__ __forceinline__ unsigned largest8(const float *v)
{
    unsigned top = mag(v[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) top = max(top, mag(v[i]));
    return top;
}

// the scale byte of a block whose largest magnitude has these fp32 bits, and the factor 2^-exponent for its values.  A mantissa above
// 1.75 (448 = 1.75 * 2^8) carries into the exponent.  An infinity or a NaN: the byte is 255, which makes every value of the block NaN.
__device__ __forceinline__ unsigned e4m3_block_scale(unsigned amax_bits, float &inv)
{
    const bool bad = amax_bits >= 0x7F800000u;
    const unsigned e = (amax_bits + 0x1FFFFFu) >> 23;           // biased exponent of the power of two, + 8
    const unsigned byte = bad ? 255u : e < 8 ? 0u : e - 8;
    inv = bad ? 0.f : __uint_as_float((254u - byte) << 23);     // 2^(127 - byte): byte 0 .. 247
    return byte;
}

// eight values times inv -> eight codes, to nearest even (in a block of scale 255, whose inv is 0: zeros)
__device__ __forceinline__ uint2 e4m3_codes8(const float *v, float inv)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i] * inv;
    int a = 0, b = 0;
    a = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], a, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], b, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], b, true);
    return inv == 0.f ? make_uint2(0u, 0u) : make_uint2((unsigned)a, (unsigned)b);
}

// largest of 16 neighbouring lanes' values, in all of them
__device__ __forceinline__ unsigned max16(unsigned x)
{
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));       // quad_perm [1,0,3,2]
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));       // quad_perm [2,3,0,1]
    x = max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xF, 0xF, true));      // row_ror:4
    return max(x, (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xF, 0xF, true));   // row_ror:8
}

}  // namespace svg2

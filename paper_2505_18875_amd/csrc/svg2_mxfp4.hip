// Microscaled 4-bit floating point (OCP MXFP4): quantisation, the values back, and the product C = A B^T + bias.
//
// A block of 32 values along the contracted axis shares one power of two (E8M0: exponent + 127, 255 is NaN); a value is E2M1:
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign.  Exponent of a block: floor(log2(amax)) - 2, so that its largest value lands in
// [4, 8) and saturates at 6; rounding to nearest, ties to the even code.  Storage of R rows and K columns, Kp = K rounded up to
// 128 (the columns behind K are zeros): codes [R, Kp/2], element 2j in the low half of byte j; scales [Kp/128, R, 4].  A row's
// four scales of 128 columns are one word, and the words of neighbouring rows are neighbours: what a tile of the product needs
// of them is one contiguous load.
#include "svg2_common.h"

namespace svg2 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return bf16_to_f32(x); }

// two fp32 -> two bf16, to nearest even (NaN stays NaN)
__device__ __forceinline__ unsigned pack_bf16(float a, float b)
{
    const f32x2 p = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
}

// the scale byte of a block whose largest magnitude has these fp32 bits, and the factor 2^-exponent for its values.  Infinities
// and NaN have no block exponent: the byte is 255, which makes every value of the block NaN.
__device__ __forceinline__ unsigned block_scale(unsigned amax_bits, float &inv)
{
    int e = (int)(amax_bits >> 23);             // biased exponent; 0: zero or subnormal, far below the smallest scale
    const unsigned byte = e == 255 ? 255u : (unsigned)(e < 2 ? 0 : e - 2);
    inv = e == 255 ? 0.f : __uint_as_float((254u - byte) << 23);        // 2^(127 - byte): byte 0 .. 252
    return byte;
}

// eight values times inv -> eight codes
__device__ __forceinline__ unsigned codes8(const float *v, float inv)
{
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * inv, v[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inv, v[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * inv, v[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * inv, v[7] * inv, 1.0f, 3);
    return w;
}

// |x| as bits: they order like the magnitudes, NaN above infinity
__device__ __forceinline__ unsigned mag(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

struct QuantArgs {
    const void *X;
    long long sm, sg;               // strides of rows and of groups of columns
    int M, G, Kg;                   // X is [M, G, Kg]; K = G Kg columns
    uint8_t *codes, *scales;
};

template <typename T> __device__ __forceinline__ const T *element(const QuantArgs &A, long long m, int k)
{
    const int g = A.G == 1 ? 0 : k / A.Kg;
    return static_cast<const T *>(A.X) + m * A.sm + g * A.sg + (k - g * A.Kg);
}

// eight neighbouring columns; VEC: 16-byte loads (the caller has checked strides and alignment, and that 8 divides Kg)
template <typename T, bool VEC> __device__ __forceinline__ void load8(const QuantArgs &A, long long m, int k, int K, float *v)
{
    if constexpr (VEC) {
        if (k >= K) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
            return;
        }
        const uint4 *p = reinterpret_cast<const uint4 *>(element<T>(A, m, k));
        if constexpr (sizeof(T) == 4) {
            const uint4 a = p[0], b = p[1];
            const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            const uint4 a = p[0];
            const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < K ? to_f32(*element<T>(A, m, k + i)) : 0.f;
    }
}

// rows: grid (ceil(M / 16), slices of the columns), block 256: 16 lanes a row of 128 columns, 4 lanes a block of 32
template <typename T, bool VEC> __global__ __launch_bounds__(256) void mxfp4_quant_kernel(const QuantArgs A)
{
    const int lane16 = threadIdx.x & 15, K = A.G * A.Kg, nk = (K + 127) / 128;
    const long long m = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (m >= A.M) return;                       // whole groups of 16 lanes: the exchanges below stay inside 4
    for (int kc = blockIdx.y; kc < nk; kc += gridDim.y) {
        float v[8];
        load8<T, VEC>(A, m, kc * 128 + lane16 * 8, K, v);
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, mag(v[i]));
        top = max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));     // quad_perm [1,0,3,2]
        top = max(top, (unsigned)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true));     // quad_perm [2,3,0,1]
        float inv;
        const unsigned byte = block_scale(top, inv);
        if (byte == 255)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        reinterpret_cast<unsigned *>(A.codes + m * (nk * 64LL) + kc * 64)[lane16] = codes8(v, inv);
        if ((lane16 & 3) == 0) A.scales[((long long)kc * A.M + m) * 4 + (lane16 >> 2)] = (uint8_t)byte;
    }
}

// transposed: the rows of the result are the columns of X, blocks run along the rows of X.
// grid (ceil(K / 64), slices of the rows), block 256: tiles of 128 rows x 64 columns through LDS; four lanes a column, 32 rows
// each.  Row m of the tile starts at word 33 m (bf16; 65 m in fp32) plus 8 words for each 32 rows before it, so that the 64 lanes
// of a wavefront, 16 columns x 4 blocks, read every bank once (fp32: twice, as the 256 bytes must).
template <typename T, bool VEC> __global__ __launch_bounds__(256) void mxfp4_quant_t_kernel(const QuantArgs A)
{
    constexpr int ROW = 64 + 4 / sizeof(T), PAD = 32 / sizeof(T);
    __shared__ T tile[128 * ROW + 4 * PAD];
    const int K = A.G * A.Kg, nm = (A.M + 127) / 128, r0 = blockIdx.x * 64;
    const int rr = threadIdx.x >> 2, mb = threadIdx.x & 3;          // phase 2: column, block of 32 rows
    for (int mc = blockIdx.y; mc < nm; mc += gridDim.y) {
        __syncthreads();
        for (int i = threadIdx.x; i < 128 * 8; i += 256) {
            const int m = i >> 3, c = (i & 7) * 8;
            const long long gm = (long long)mc * 128 + m;
            float v[8];
            if (gm < A.M) load8<T, VEC>(A, gm, r0 + c, K, v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
            T *row = tile + m * ROW + (m >> 5) * PAD + c;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (sizeof(T) == 4) row[e] = v[e];
                else row[e] = (bf16_t)(__float_as_uint(v[e]) >> 16);
            }
        }
        __syncthreads();
        float v[32];
        unsigned top = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            v[e] = to_f32(tile[(mb * 32 + e) * ROW + mb * PAD + rr]);
            top = max(top, mag(v[e]));
        }
        float inv;
        const unsigned byte = block_scale(top, inv);
        if (byte == 255)
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0.f;
        if (r0 + rr < K) {
            const long long r = r0 + rr;
            *reinterpret_cast<uint4 *>(A.codes + r * (nm * 64LL) + mc * 64 + mb * 16) =
                make_uint4(codes8(v, inv), codes8(v + 8, inv), codes8(v + 16, inv), codes8(v + 24, inv));
            A.scales[((long long)mc * K + r) * 4 + mb] = (uint8_t)byte;
        }
    }
}

// ---- the values back -------------------------------------------------------
// 2^(byte - 127) in two factors, neither of which leaves the normal range; byte 255 is NaN
__device__ __forceinline__ void scale_factors(unsigned byte, float &a, float &b)
{
    const unsigned half = byte >> 1;
    a = byte == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float((half + 64) << 23);       // 2^(half - 63)
    b = __uint_as_float((byte - half + 63) << 23);                                             // 2^(byte - half - 64)
}

// grid (ceil(M / 16), slices of the columns), block 256: 8 values a lane; VEC: 16-byte stores
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void mxfp4_values_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                           int M, int K, T *__restrict__ X, long long ldx)
{
    const int lane16 = threadIdx.x & 15, nk = (K + 127) / 128;
    const long long m = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (m >= M) return;
    for (int kc = blockIdx.y; kc < nk; kc += gridDim.y) {
        const unsigned w = reinterpret_cast<const unsigned *>(codes + m * (nk * 64LL) + kc * 64)[lane16];
        float a, b, v[8];
        scale_factors(scales[((long long)kc * M + m) * 4 + (lane16 >> 2)], a, b);
        const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[i >> 1][i & 1] * a * b;
        const int k = kc * 128 + lane16 * 8;
        T *x = X + m * ldx + k;
        unsigned u[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        if (VEC && k + 8 <= K) {
            if constexpr (sizeof(T) == 4) {
                reinterpret_cast<float4 *>(x)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4 *>(x)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                *reinterpret_cast<uint4 *>(x) = make_uint4(u[0], u[1], u[2], u[3]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < K) {
                    if constexpr (sizeof(T) == 4) x[i] = v[i];
                    else x[i] = (bf16_t)(u[i >> 1] >> (16 * (i & 1)));
                }
        }
    }
}

// ---- the product -----------------------------------------------------------
struct ProductArgs {
    const uint8_t *A, *B, *SA, *SB; // codes [M, Kp/2], [N, Kp/2]; scales [Kp/128, M, 4], [Kp/128, N, 4]
    int M, N, nk;                   // nk = Kp / 128
    const float *bias;
    void *C;
    long long ldc;
    int tiles_n;
};

template <typename T> __device__ __forceinline__ void store4(T *c, const float *v, int left, bool vec)
{
    if constexpr (sizeof(T) == 4) {
        if (vec && left >= 4) { *reinterpret_cast<float4 *>(c) = make_float4(v[0], v[1], v[2], v[3]); return; }
    } else {
        if (vec && left >= 4) { *reinterpret_cast<uint2 *>(c) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])); return; }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) {
            if constexpr (sizeof(T) == 4) c[i] = v[i];
            else c[i] = (bf16_t)pack_bf16(v[i], 0.f);
        }
}

// v_mfma_scale_f32_32x32x64_f8f6f4 on E2M1 operands: lane l gives 32 values of row l % 32 (16 bytes), columns 32 (l / 32) ..,
// and their scale.  The rows of B go in first: a lane's results are then neighbours in a row of C.
// grid (tiles), block 256 = 2 x 2 wavefronts of 64 x 64 results; rows behind the last are read as the last and not stored.
template <typename T> __global__ __launch_bounds__(256) void mxfp4_product_kernel(const ProductArgs P, bool vec)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 31, half = lane >> 5;
    const int m0 = (blockIdx.x / P.tiles_n) * 128 + (wave >> 1) * 64, n0 = (blockIdx.x % P.tiles_n) * 128 + (wave & 1) * 64;
    f32x16 acc[2][2] = {};
    const uint8_t *a[2], *b[2];
    const unsigned *sa[2], *sb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int m = min(m0 + 32 * i + row, P.M - 1), n = min(n0 + 32 * i + row, P.N - 1);
        a[i] = P.A + (long long)m * P.nk * 64 + half * 16;
        b[i] = P.B + (long long)n * P.nk * 64 + half * 16;
        sa[i] = reinterpret_cast<const unsigned *>(P.SA) + m;
        sb[i] = reinterpret_cast<const unsigned *>(P.SB) + n;
    }
    for (int kc = 0; kc < P.nk; ++kc) {
        int xa[2], xb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            xa[i] = (int)(sa[i][(long long)kc * P.M] >> (8 * half));        // bytes 0 and 2: this half's blocks
            xb[i] = (int)(sb[i][(long long)kc * P.N] >> (8 * half));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            i32x8 fa[2], fb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int4 u = *reinterpret_cast<const int4 *>(a[i] + kc * 64LL + k * 32), w = *reinterpret_cast<const int4 *>(b[i] + kc * 64LL + k * 32);
                fa[i] = i32x8{u.x, u.y, u.z, u.w, 0, 0, 0, 0};
                fb[i] = i32x8{w.x, w.y, w.z, w.w, 0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = k == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[i], acc[i][j], 4, 4, 0, xb[j], 0, xa[i])
                                       : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[i], acc[i][j], 4, 4, 2, xb[j], 2, xa[i]);
        }
    }
    // results: lane holds row m0 + 32 i + l % 32 of C, columns n0 + 32 j + 8 q + 4 (l / 32) .. + 3 in registers 4 q .. 4 q + 3
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int m = m0 + 32 * i + row;
        if (m >= P.M) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + 32 * j + 8 * q + 4 * half;
                if (n >= P.N) continue;
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r] + (P.bias && n + r < P.N ? P.bias[n + r] : 0.f);
                store4(static_cast<T *>(P.C) + (long long)m * P.ldc + n, v, P.N - n, vec);
            }
    }
}

// ---- launchers -------------------------------------------------------------
// slices of a loop so that there are some 2048 workgroups, where the loop has that many steps
static int slices(long long blocks, int steps)
{
    const long long want = (2048 + blocks - 1) / blocks;
    return (int)(want < 1 ? 1 : want > steps ? steps : want);
}

static bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int mxfp4_quant_launch(const void *X, int dtype, int M, int G, int Kg, int64_t sm, int64_t sg, bool transposed, void *codes,
                       void *scales, hipStream_t st)
{
    const QuantArgs A = {X, sm, sg, M, G, Kg, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales)};
    const int K = G * Kg, per16 = dtype == SVG2_BF16 ? 8 : 4;
    const bool vec = aligned(X, 16) && sm % per16 == 0 && (G == 1 || sg % per16 == 0) && Kg % 8 == 0;
    if (!transposed) {
        const int bx = cdiv(M, 16);
        const dim3 grid(bx, slices(bx, cdiv(K, 128)));
        if (dtype == SVG2_BF16) {
            if (vec) mxfp4_quant_kernel<bf16_t, true><<<grid, 256, 0, st>>>(A);
            else mxfp4_quant_kernel<bf16_t, false><<<grid, 256, 0, st>>>(A);
        } else {
            if (vec) mxfp4_quant_kernel<float, true><<<grid, 256, 0, st>>>(A);
            else mxfp4_quant_kernel<float, false><<<grid, 256, 0, st>>>(A);
        }
    } else {
        const int bx = cdiv(K, 64);
        const dim3 grid(bx, slices(bx, cdiv(M, 128)));
        if (dtype == SVG2_BF16) {
            if (vec) mxfp4_quant_t_kernel<bf16_t, true><<<grid, 256, 0, st>>>(A);
            else mxfp4_quant_t_kernel<bf16_t, false><<<grid, 256, 0, st>>>(A);
        } else {
            if (vec) mxfp4_quant_t_kernel<float, true><<<grid, 256, 0, st>>>(A);
            else mxfp4_quant_t_kernel<float, false><<<grid, 256, 0, st>>>(A);
        }
    }
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int mxfp4_values_launch(const void *codes, const void *scales, int M, int K, int dtype, void *X, int64_t ldx, hipStream_t st)
{
    const uint8_t *c = static_cast<const uint8_t *>(codes), *s = static_cast<const uint8_t *>(scales);
    const bool vec = aligned(X, 16) && ldx % (dtype == SVG2_BF16 ? 8 : 4) == 0;
    const int bx = cdiv(M, 16);
    const dim3 grid(bx, slices(bx, cdiv(K, 128)));
    if (dtype == SVG2_BF16) {
        if (vec) mxfp4_values_kernel<bf16_t, true><<<grid, 256, 0, st>>>(c, s, M, K, static_cast<bf16_t *>(X), ldx);
        else mxfp4_values_kernel<bf16_t, false><<<grid, 256, 0, st>>>(c, s, M, K, static_cast<bf16_t *>(X), ldx);
    } else {
        if (vec) mxfp4_values_kernel<float, true><<<grid, 256, 0, st>>>(c, s, M, K, static_cast<float *>(X), ldx);
        else mxfp4_values_kernel<float, false><<<grid, 256, 0, st>>>(c, s, M, K, static_cast<float *>(X), ldx);
    }
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

size_t mxfp4_matmul_ws_bytes(int M, int N, int K) { (void)M; (void)N; (void)K; return 256; }

int mxfp4_matmul_launch(const void *A, const void *SA, const void *B, const void *SB, int M, int N, int K, const float *bias,
                        int out_dtype, void *C, int64_t ldc, void *ws, hipStream_t st)
{
    (void)ws;
    ProductArgs P = {static_cast<const uint8_t *>(A), static_cast<const uint8_t *>(B), static_cast<const uint8_t *>(SA),
                     static_cast<const uint8_t *>(SB), M, N, cdiv(K, 128), bias, C, ldc, cdiv(N, 128)};
    const bool vec = aligned(C, out_dtype == SVG2_BF16 ? 8 : 16) && ldc % 4 == 0;
    const int tiles = cdiv(M, 128) * P.tiles_n;
    if (out_dtype == SVG2_BF16) mxfp4_product_kernel<bf16_t><<<tiles, 256, 0, st>>>(P, vec);
    else mxfp4_product_kernel<float><<<tiles, 256, 0, st>>>(P, vec);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

}  // namespace svg2

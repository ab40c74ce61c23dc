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

// 4 bytes per lane into LDS (see load_to_lds_16)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds_4(const char *base, unsigned byte_off, const unsigned char *dst)
{
    const unsigned lds_addr = (unsigned)(size_t)(const lds_u8 *)dst;
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
                 :
                 : "v"(byte_off), "s"(base), "s"(lds_addr)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

__device__ __forceinline__ i32x8 fragment(const uint4 &u) { return i32x8{(int)u.x, (int)u.y, (int)u.z, (int)u.w, 0, 0, 0, 0}; }

// The tiled product.  v_mfma_scale_f32_32x32x64_f8f6f4 on E2M1 operands: lane l gives 32 values of row l % 32 (16 bytes), columns
// 32 (l / 32) .., and their scale.  The rows of B go in first: a lane's results are then neighbours in a row of C.
//
// Workgroup: 2 x 2 wavefronts of 32 WT x 32 WT results, one tile of C after another.  A stage is 128 columns of the 64 WT rows of
// either side with their scales; NB stages are in LDS, all but one of them on their way while one is used, straight from memory
// (global_load_lds).  Within a stage the two halves of 64 columns alternate between two register sets: the next half is read from
// LDS while the matrix instructions of this one run.  The one barrier of a stage stands in its middle.
// WT = 4, one wavefront a SIMD: 32 instructions of 32 cycles a stage, in which LDS gives 64 KB to the registers (512 cycles) and
// takes 34 KB (272).
// In LDS row r has 64 bytes, its 16-byte piece c at c ^ spread(r): eight neighbouring rows then take every bank once.
// Rows behind the last are read as the last and not stored.
template <int WT> struct Tile {
    static constexpr int BT = 64 * WT, SIDE = BT * 64, STAGE = 2 * SIDE + 2 * BT * 4;
    static constexpr int NB = WT == 4 ? 4 : 3;                              // stages in LDS
    static constexpr int NS = WT < 2 ? 1 : WT / 2, LOADS = 2 * WT + NS;     // loads of a wavefront and stage: scales, all
    // results on their way out: 32 rows of 128 bytes (WT = 1, bf16: 64) for each wavefront
    template <typename T> static constexpr int out_cols() { return 32 * WT * (int)sizeof(T) < 128 ? 32 * WT : 128 / (int)sizeof(T); }
    template <typename T> static constexpr int out_row() { return out_cols<T>() * (int)sizeof(T) + 16; }
    static constexpr int BIAS = NB * STAGE, OUT = BIAS + 2 * BT * 4;
    template <typename T> static constexpr int lds() { return OUT + 4 * 32 * out_row<T>(); }
};

__device__ __forceinline__ int spread(int r) { return ((r >> 1) & 3) ^ ((r >> 3) & 1); }

template <int WT, typename T> __global__ __launch_bounds__(256, WT == 4 ? 1 : 2) void mxfp4_product_kernel(const ProductArgs P, bool vec)
{
    using L = Tile<WT>;
    constexpr int BT = L::BT, SIDE = L::SIDE, STAGE = L::STAGE, NB = L::NB, NS = L::NS, LOADS = L::LOADS, MULS = WT * WT;
    extern __shared__ __attribute__((aligned(256))) unsigned char s_tile[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 31, half = lane >> 5;
    const long long row_bytes = (long long)P.nk * 64;
    const int nk = P.nk;

    // Which tiles: the XCDs (every eighth workgroup) get contiguous parts of an order that goes down 8 tiles of C, then right, and
    // their workgroups take turns, so that what an XCD works on at a time is a compact patch and shares its rows in that XCD's L2.
    const int tiles_m = (P.M + BT - 1) / BT, total = tiles_m * P.tiles_n;
    const int xcd = blockIdx.x & 7, part = total >> 3, rest = total & 7, first = xcd * part + min(xcd, rest);
    const int mine = part + (xcd < rest), slots = (gridDim.x + 7 - xcd) >> 3;

    int m0, n0;
    const char *ga, *gb, *gsa, *gsb;
    unsigned off_a[WT], off_b[WT], off_s[NS];           // this lane's part of the loads: 16 rows x 64 bytes each
    auto set_tile = [&](int k) {
        const int t = first + k, group = t / (8 * P.tiles_n), in = t - group * 8 * P.tiles_n, high = min(8, tiles_m - group * 8);
        m0 = (group * 8 + in % high) * BT;
        n0 = (in / high) * BT;
        ga = reinterpret_cast<const char *>(P.A) + m0 * row_bytes;
        gb = reinterpret_cast<const char *>(P.B) + n0 * row_bytes;
        gsa = reinterpret_cast<const char *>(P.SA) + m0 * 4LL;
        gsb = reinterpret_cast<const char *>(P.SB) + n0 * 4LL;
        int l = lane;
        asm("" : "+v"(l));
#pragma unroll
        for (int i = 0; i < WT; ++i) {
            const int r = (wave * WT + i) * 16 + (l >> 2), piece = (l & 3) ^ spread(r);
            off_a[i] = (unsigned)min(r, P.M - 1 - m0) * (unsigned)row_bytes + piece * 16;
            off_b[i] = (unsigned)min(r, P.N - 1 - n0) * (unsigned)row_bytes + piece * 16;
        }
        // scales: 2 BT words, A's then B's, 64 a load (WT = 1: two wavefronts load the same)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int at = (wave * NS + i) * 64 % (2 * BT), r = at % BT + l;
            off_s[i] = 4u * (unsigned)(at < BT ? min(r, P.M - 1 - m0) : min(r, P.N - 1 - n0));
        }
    };
    // piece g of a stage's loads: WT of A, WT of B, NS of scales
    auto load_piece = [&](int kc, int g) {
        unsigned char *to = s_tile + (kc % NB) * STAGE;
        if (g < WT) {
            load_to_lds_16(ga + kc * 64LL, off_a[g], to + (wave * WT + g) * 1024);
        } else if (g < 2 * WT) {
            load_to_lds_16(gb + kc * 64LL, off_b[g - WT], to + SIDE + (wave * WT + g - WT) * 1024);
        } else {
            const int at = (wave * NS + g - 2 * WT) * 64 % (2 * BT);
            load_to_lds_4(at < BT ? gsa + kc * 4LL * P.M : gsb + kc * 4LL * P.N, off_s[g - 2 * WT], to + 2 * SIDE + at * 4);
        }
    };
    // what a tile's first NB - 1 stages need, its bias in front (WT < 4: some wavefronts load the same part)
    auto load_first = [&](int copy) {
        if (P.bias)
            load_to_lds_4(reinterpret_cast<const char *>(P.bias + n0), 4u * (unsigned)min(wave * 64 % BT + lane, P.N - 1 - n0),
                          s_tile + L::BIAS + copy * BT * 4 + wave * 64 % BT * 4);
#pragma unroll
        for (int kc = 0; kc < NB - 1; ++kc)
            if (kc < nk)
#pragma unroll
                for (int g = 0; g < LOADS; ++g) load_piece(kc, g);
    };

    f32x16 acc[WT][WT];
    const int ra = (wave >> 1) * 32 * WT, rb = (wave & 1) * 32 * WT;
    const int at = row * 64 + ((half ^ spread(row)) << 4);          // first half of a stage; the second: piece ^ 2
    struct Set { uint4 a[WT], b[WT]; };
    // fragment g of a half: b 0, a 0, b 1 .., a 1 ..: in the order in which the products need them
    auto read_piece = [&](int kc, int k, int g, Set &f) {
        const unsigned char *s = s_tile + (kc % NB) * STAGE + (at ^ (k * 32));
        const bool is_a = g == 1 || g > WT;
        const int i = g < 2 ? 0 : g <= WT ? g - 1 : g - WT;
        if (is_a) f.a[i] = *reinterpret_cast<const uint4 *>(s + (ra + 32 * i) * 64);
        else f.b[i] = *reinterpret_cast<const uint4 *>(s + SIDE + (rb + 32 * i) * 64);
    };
    struct Scales { unsigned a[WT], b[WT]; };
    auto read_scales = [&](int kc, Scales &x) {
        const unsigned *s = reinterpret_cast<const unsigned *>(s_tile + (kc % NB) * STAGE + 2 * SIDE);
#pragma unroll
        for (int i = 0; i < WT; ++i) {
            x.b[i] = s[BT + rb + 32 * i + row];
            x.a[i] = s[ra + 32 * i + row];
        }
    };
    auto take_scales = [&](const Scales &x, Scales &y) {            // bytes 0 and 2: this lane's blocks of the two halves
#pragma unroll
        for (int i = 0; i < WT; ++i) {
            y.a[i] = x.a[i] >> (8 * half);
            y.b[i] = x.b[i] >> (8 * half);
        }
    };
    auto multiply = [&](const Set &f, const Scales &x, int e, auto second) {
        constexpr int SEL = decltype(second)::value ? 2 : 0;
        const int i = e / WT, j = e % WT;
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fragment(f.b[j]), fragment(f.a[i]), acc[i][j], 4, 4, SEL,
                                                                    (int)x.b[j], SEL, (int)x.a[i]);
    };

    // Loads and stores come back in the order in which they were issued.  The last tile's stores lie between the loads of this
    // tile's first NB - 1 stages and all later ones, and the first waits of a tile let them pass (`after`: that many were issued).
    constexpr int STORES = WT * WT * 32 * 32 * (int)sizeof(T) / 1024;
    bool after = false;
    auto wait_but = [&](auto loads, bool stores) {
        constexpr int N = decltype(loads)::value;
        if (stores) wait_loads<(N + STORES < 63 ? N + STORES : 63)>();
        else wait_loads<N>();
    };

    Set f0, f1;
    Scales x, next;
    // One stage.  NEXT: there is a stage behind it; LOAD: and one NB - 1 behind it; PENDING: loads that may still be on their way when
    // stage kc + 1 is needed.  Between the fences the written order is kept, LDS reads and loads spread over the matrix instructions:
    // left to itself the compiler puts all reads in front and the matrix cores wait for them.
    auto step = [&](int kc, auto load, auto has_next, auto pending) {
        constexpr bool LOAD = decltype(load)::value, NEXT = decltype(has_next)::value;
        constexpr int READS = 2 * WT, LOADS_FROM = MULS > LOADS ? MULS - LOADS : 0;
#pragma unroll
        for (int e = 0; e < (MULS > READS ? MULS : READS); ++e) {
            if (e < READS) read_piece(kc, 1, e, f1);
            if (e < MULS) multiply(f0, x, e, std::false_type());
            __builtin_amdgcn_sched_barrier(0);
        }
        if (NEXT) {
            // stage kc + 1 has arrived for every wavefront; every wavefront is done with stage kc - 1, whose place is free
            wait_but(pending, after && kc < NB - 2);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            read_scales(kc + 1, next);
        }
#pragma unroll
        for (int e = 0; e < (MULS > READS ? MULS : READS); ++e) {
            if (NEXT && e < READS) read_piece(kc + 1, 0, e, f0);
            if (LOAD) {
                if (MULS > LOADS) {
                    if (e >= LOADS_FROM) load_piece(kc + NB - 1, e - LOADS_FROM);
                } else {
#pragma unroll
                    for (int g = 0; g < LOADS; ++g)
                        if (g * READS / LOADS == e) load_piece(kc + NB - 1, g);
                }
            }
            if (e < MULS) multiply(f1, x, e, std::true_type());
            __builtin_amdgcn_sched_barrier(0);
        }
        if (NEXT) take_scales(next, x);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    using Most = std::integral_constant<int, (NB - 3) * LOADS>;
    using None = std::integral_constant<int, 0>;

    int k = blockIdx.x >> 3, copy = 0;
    if (k >= mine) return;
    set_tile(k);
    load_first(copy);
    for (; k < mine; k += slots, copy ^= 1) {
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j = 0; j < WT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        if (nk >= NB - 1) wait_but(std::integral_constant<int, (NB - 2) * LOADS>(), after);
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read_scales(0, next);
#pragma unroll
        for (int g = 0; g < 2 * WT; ++g) read_piece(0, 0, g, f0);
        take_scales(next, x);
        int kc = 0;
        for (; kc + NB - 1 < nk; ++kc) step(kc, Yes(), Yes(), Most());
        if (NB > 3 && kc + 2 < nk) step(kc++, No(), Yes(), Most());
        for (; kc + 1 < nk; ++kc) step(kc, No(), Yes(), None());
        step(kc, No(), No(), None());
        __builtin_amdgcn_s_barrier();                               // every wavefront has read its last stage
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");         // the last results are read by vector instructions from here on

        const int m_first = m0 + ra, n_first = n0 + rb, n_left = P.N - n_first;
        const bool full = vec && m0 + BT <= P.M && n0 + BT <= P.N;
        if (k + slots < mine) {                                     // the next tile's first stages come while this one goes out
            set_tile(k + slots);
            load_first(copy ^ 1);
        }
        after = full;

        // Results: lane holds row m_first + 32 i + l % 32 of C, columns n_first + 32 j + 8 q + 4 (l / 32) .. + 3 in registers 4 q ..
        // 4 q + 3.  Stored from there, an instruction would write 32 pieces of 16 bytes; 32 rows of 128 bytes at a time go through LDS
        // instead (a part of its own for each wavefront).
        constexpr int COLS = L::template out_cols<T>(), ROW = L::template out_row<T>(), PER16 = 16 / (int)sizeof(T), JS = COLS / 32;
        int l = lane;
        asm("" : "+v"(l));         // addresses below are formed here, not kept in registers through the loop over the stages
        unsigned char *s = s_tile + L::OUT + wave * 32 * ROW;
        const float *bias = reinterpret_cast<const float *>(s_tile + L::BIAS) + copy * BT + rb;
#pragma unroll
        for (int i = 0; i < WT; ++i)
#pragma unroll
            for (int j0 = 0; j0 < WT; j0 += JS) {
#pragma unroll
                for (int j = j0; j < j0 + JS; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int n = 32 * j + 8 * q + 4 * (l >> 5);
                        float v[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r];
                        if (P.bias) {
                            const float4 add = *reinterpret_cast<const float4 *>(bias + n);
                            v[0] += add.x; v[1] += add.y; v[2] += add.z; v[3] += add.w;
                        }
                        unsigned char *to = s + (l & 31) * ROW + (n - 32 * j0) * (int)sizeof(T);
                        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
                        else *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                    }
                constexpr int LANES = COLS / PER16, AT_ONCE = 64 / LANES;       // lanes a row, rows an instruction
                T *C = static_cast<T *>(P.C) + (long long)(m_first + 32 * i) * P.ldc + n_first + 32 * j0;
                const int rows = P.M - m_first - 32 * i, cols = n_left - 32 * j0;
                if (full) {
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += AT_ONCE) {
                        const int r = r0 + l / LANES, c = l % LANES;
                        *reinterpret_cast<uint4 *>(C + (long long)r * P.ldc + c * PER16) = *reinterpret_cast<const uint4 *>(s + r * ROW + c * 16);
                    }
                } else {
                    for (int e = l; e < 32 * COLS; e += 64) {
                        const int r = e / COLS, c = e % COLS;
                        if (r < rows && c < cols) C[(long long)r * P.ldc + c] = reinterpret_cast<const T *>(s + r * ROW)[c];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);      // else all results leave the accumulators first, for want of registers to memory
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

template <int WT> static int prepare_tiles()
{
    SVG2_TRY(set_dynamic_lds(reinterpret_cast<const void *>(&mxfp4_product_kernel<WT, bf16_t>), Tile<WT>::template lds<bf16_t>()));
    return set_dynamic_lds(reinterpret_cast<const void *>(&mxfp4_product_kernel<WT, float>), Tile<WT>::template lds<float>());
}

int mxfp4_matmul_prepare()
{
    SVG2_TRY(prepare_tiles<4>());
    SVG2_TRY(prepare_tiles<2>());
    return prepare_tiles<1>();
}

template <int WT> static int product_tiles(ProductArgs P, int out_dtype, bool vec, hipStream_t st)
{
    P.tiles_n = cdiv(P.N, 64 * WT);
    const int tiles = cdiv(P.M, 64 * WT) * P.tiles_n, resident = 256 * (WT == 4 ? 1 : WT == 2 ? 2 : 4);
    const int grid = tiles < resident ? tiles : resident;
    if (out_dtype == SVG2_BF16) mxfp4_product_kernel<WT, bf16_t><<<grid, 256, Tile<WT>::template lds<bf16_t>(), st>>>(P, vec);
    else mxfp4_product_kernel<WT, float><<<grid, 256, Tile<WT>::template lds<float>(), st>>>(P, vec);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int mxfp4_matmul_launch(const void *A, const void *SA, const void *B, const void *SB, int M, int N, int K, const float *bias,
                        int out_dtype, void *C, int64_t ldc, void *ws, hipStream_t st)
{
    (void)ws;
    const ProductArgs P = {static_cast<const uint8_t *>(A), static_cast<const uint8_t *>(B), static_cast<const uint8_t *>(SA),
                           static_cast<const uint8_t *>(SB), M, N, cdiv(K, 128), bias, C, ldc, 0};
    const bool vec = aligned(C, 16) && ldc % (out_dtype == SVG2_BF16 ? 8 : 4) == 0;
    // the largest tile that leaves every CU one
    auto tiles = [&](int wt) { return (long long)cdiv(M, 64 * wt) * cdiv(N, 64 * wt); };
    if (tiles(4) >= 256) return product_tiles<4>(P, out_dtype, vec, st);
    if (tiles(2) >= 256) return product_tiles<2>(P, out_dtype, vec, st);
    return product_tiles<1>(P, out_dtype, vec, st);
}

}  // namespace svg2

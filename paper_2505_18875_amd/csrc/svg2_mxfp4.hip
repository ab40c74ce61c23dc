// Microscaled 4-bit floating point (OCP MXFP4): quantisation, the values back, and the product C = A B^T + bias.
//
// A block of 32 values along the contracted axis shares one power of two (E8M0: exponent + 127, 255 is NaN); a value is E2M1:
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign.  Exponent of a block: floor(log2(amax)) - 2, so that its largest value lands in
// [4, 8) and saturates at 6; rounding to nearest, ties to the even code.  Storage of R rows and K columns, Kp = K rounded up to
// 128 (the columns behind K are zeros): codes [R, Kp/2], element 2j in the low half of byte j; scales [Kp/128, R, 4].  A row's
// four scales of 128 columns are one word, and the words of neighbouring rows are neighbours: what a tile of the product needs
// of them is one contiguous load.
#include <type_traits>

#include "svg2_common.h"

namespace svg2 {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));     // 16 bytes at any element's address: one load or store all the same
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;

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

// eight neighbouring columns: one load where they are all there and in one group, whatever their address; STREAM: past the caches,
// for an X that is larger than they are (see streamed)
template <typename T, bool STREAM> __device__ __forceinline__ void load8(const QuantArgs &A, long long m, int k, int K, float *v)
{
    if (k + 8 <= K && (A.G == 1 || k % A.Kg + 8 <= A.Kg)) {
        const u32x4_any *p = reinterpret_cast<const u32x4_any *>(element<T>(A, m, k));
        const u32x4 a = STREAM ? __builtin_nontemporal_load(p) : *p;
        if constexpr (sizeof(T) == 4) {
            const u32x4 b = STREAM ? __builtin_nontemporal_load(p + 1) : p[1];
            const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
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

// rows: grid (ceil(M / 16), slices of the columns), block 256: 16 lanes a row of 128 columns, 4 lanes a block of 32.  A value is read
// once, a lane's eight stay in registers, and a block's maximum goes round four neighbouring lanes without LDS.  Bound by HBM:
// 75,600 x 5120 bf16 (774 MB in, 206 out) 180 to 192 us, 5.1 to 5.4 TB/s; 75,599 x 5119, whose rows share lines, 236.
template <typename T, bool STREAM> __global__ __launch_bounds__(256) void mxfp4_quant_kernel(const QuantArgs A)
{
    const int lane16 = threadIdx.x & 15, K = A.G * A.Kg, nk = (K + 127) / 128;
    const long long m = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (m >= A.M) return;                       // whole groups of 16 lanes: the exchanges below stay inside 4
    for (int kc = blockIdx.y; kc < nk; kc += gridDim.y) {
        float v[8];
        load8<T, STREAM>(A, m, kc * 128 + lane16 * 8, K, v);
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
// grid (ceil(K / 64) rounded up to 8, slices of the rows), block 256: tiles of 128 rows x 64 columns through LDS; four lanes a column,
// 32 rows each.  A slice is `per` neighbouring tiles, an even number: two of them fill a cache line of codes.  Neighbouring columns go to
// the same XCD (every eighth workgroup): where rows are not whole lines they share some.
// Bound by HBM where X is large (75,600 x 5120 bf16: 240 us, 4.1 TB/s; 75,599 x 5119, whose rows share lines, 401), by its few long steps where
// it is small (16,384 x 1536: 14 us; 1021 x 777 fp32: 7 us, 52 workgroups with two tiles each, one after the other).
// In LDS a row takes 33 words in bf16 (65 in fp32), and 8 words more for each 32 rows before it, so that the 64 lanes of a wavefront,
// 16 columns x 4 blocks, read every bank once (fp32: twice, as the 256 bytes must).
template <typename T, bool STREAM> __global__ __launch_bounds__(256) void mxfp4_quant_t_kernel(const QuantArgs A, int per)
{
    constexpr int WORDS = 16 * (int)sizeof(T) + 1, PAD = 8;
    __shared__ unsigned tile[128 * WORDS + 4 * PAD];
    const int K = A.G * A.Kg, nm = (A.M + 127) / 128, r0 = ((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) * 64;
    const int from = blockIdx.y * per, end = r0 < K ? min(nm, from + per) : from;
    const int rr = threadIdx.x >> 2, mb = threadIdx.x & 3;          // column and block of 32 rows
    for (int mc = from; mc < end; ++mc) {
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long m = (long long)mc * 128 + i * 32 + (threadIdx.x >> 3);
            if (m < A.M) load8<T, STREAM>(A, m, r0 + (threadIdx.x & 7) * 8, K, v[i]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
        __syncthreads();                        // the last tile has been read
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned *w = tile + (i * 32 + (threadIdx.x >> 3)) * WORDS + i * PAD + (threadIdx.x & 7) * 2 * (int)sizeof(T);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(v[i][e]);
                else if (e & 1) w[e >> 1] = (__float_as_uint(v[i][e]) & 0xFFFF0000u) | (__float_as_uint(v[i][e - 1]) >> 16);
            }
        }
        __syncthreads();
        float x[32];
        unsigned top = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            x[e] = to_f32(reinterpret_cast<const T *>(tile + (mb * 32 + e) * WORDS + mb * PAD)[rr]);
            top = max(top, mag(x[e]));
        }
        float inv;
        const unsigned byte = block_scale(top, inv);
        if (byte == 255)
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = 0.f;
        const long long r = r0 + rr;
        if (r < K) {
            *reinterpret_cast<uint4 *>(A.codes + r * (nm * 64LL) + mc * 64 + mb * 16) =
                make_uint4(codes8(x, inv), codes8(x + 8, inv), codes8(x + 16, inv), codes8(x + 24, inv));
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

// grid (row groups, slices of the columns), block 256: a lane writes 16 bytes, 8 or 4 values.  Bound by the writes: 75,600 x 5120 bf16 in
// 145 us, 5.3 TB/s of values, the codes from the last cache where they were written just before.  Rows that are not whole lines: the steps of
// 256 bytes begin inside a line, so lines are written in two pieces, 75,599 x 5119 in 312 us.
template <typename T> constexpr int values_rows() { return 256 / (128 * (int)sizeof(T) / 16); }     // rows of a workgroup: 16 bf16, 8 fp32

template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void mxfp4_values_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                           int M, int K, T *__restrict__ X, long long ldx)
{
    constexpr int PER = 16 / (int)sizeof(T), LANES = 128 / PER;
    const int lane = threadIdx.x % LANES, nk = (K + 127) / 128;
    const long long m = (long long)blockIdx.x * values_rows<T>() + threadIdx.x / LANES;
    if (m >= M) return;
    for (int kc = blockIdx.y; kc < nk; kc += gridDim.y) {
        const uint8_t *from = codes + m * (nk * 64LL) + kc * 64 + lane * (PER / 2);
        const unsigned w = PER == 8 ? *reinterpret_cast<const unsigned *>(from) : *reinterpret_cast<const unsigned short *>(from);
        float a, b, v[PER];
        scale_factors(scales[((long long)kc * M + m) * 4 + lane / (32 / PER)], a, b);
        f32x2 p[4];
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
        if (PER == 8) {
            p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
            p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
        }
        unsigned u[4];
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = p[i >> 1][i & 1] * a * b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(v[i]);
            else u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        }
        const int k = kc * 128 + lane * PER;
        T *x = X + m * ldx + k;
        if (k + PER <= K) {
            const u32x4 y = {u[0], u[1], u[2], u[3]};
            if (STREAM) __builtin_nontemporal_store(y, reinterpret_cast<u32x4_any *>(x));
            else *reinterpret_cast<u32x4_any *>(x) = y;
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
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
    int split, per;                 // the contraction in `split` parts of `per` stages, each with a C of its own, one behind the other
};

// 4 bytes per lane into LDS (see load_to_lds_16)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds_4(const char *base, unsigned byte_off, const unsigned char *dst)
{
    const unsigned lds_addr = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(const lds_u8 *)dst);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
                 :
                 : "v"(byte_off), "s"(base), "s"(lds_addr)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

__device__ __forceinline__ i32x8 fragment(const uint4 &u) { return i32x8{(int)u.x, (int)u.y, (int)u.z, (int)u.w, 0, 0, 0, 0}; }

// Wait states between the last matrix instructions and the vector instructions that read their results, more than either the compiler
// or the hardware asks for (they are not agreed for these instructions).  The results are operands of the statement, all of them of
// one: it stands behind every instruction that writes them and before every one that reads them, which an s_nop by itself does not.
template <int I, int J> __device__ __forceinline__ void settle(f32x16 (&a)[I][J])
{
    static_assert(I * J == 8 || I * J == 4 || I * J == 1, "");
    if constexpr (I * J == 8)
        asm volatile("s_nop 15\n\ts_nop 15" : "+v"(a[0][0]), "+v"(a[0][1]), "+v"(a[1][0]), "+v"(a[1][1]), "+v"(a[2][0]), "+v"(a[2][1]),
                     "+v"(a[3][0]), "+v"(a[3][1]));
    else if constexpr (I * J == 4) asm volatile("s_nop 15\n\ts_nop 15" : "+v"(a[0][0]), "+v"(a[0][1]), "+v"(a[1][0]), "+v"(a[1][1]));
    else asm volatile("s_nop 15\n\ts_nop 15" : "+v"(a[0][0]));
}

// The tiled product.  v_mfma_scale_f32_32x32x64_f8f6f4 on E2M1 operands: lane l gives 32 values of row l % 32 (16 bytes), columns
// 32 (l / 32) .., and their scale.  The rows of B go in first: a lane's results are then neighbours in a row of C.
//
// Workgroup: WM x WN wavefronts of 32 WI x 32 WJ results, one tile of C after another.  A stage is 256 columns of the tile's rows of
// either side with their scales: 128 bytes of a row, a cache line.  Two stages are in LDS, one on its way while the other is used,
// straight from memory (global_load_lds).  A stage is used in four quarters of 64 columns, which alternate between two register
// sets: the next quarter is read from LDS while the matrix instructions of this one run.  The one barrier of a stage stands before
// its last quarter: the next stage has arrived by then, and this one's place is free as soon as its last quarter is in registers.
// Where there are few tiles and many stages, a part of the stages is a tile of its own (split), and mxfp4_join_kernel adds them up.
// In LDS row r has 128 bytes, its 16-byte piece c at c ^ spread(r): eight neighbouring rows then take every bank once.  Bank conflicts are counted
// where results go through LDS, 1536 cycles a tile of 256 x 256 whatever the number of its stages (6.6 % of the LDS cycles at 20 stages).
// Rows behind the last are read as the last and not stored.
template <int WM_, int WN_, int WI_, int WJ_> struct Tile {
    static constexpr int WM = WM_, WN = WN_, WI = WI_, WJ = WJ_, WAVES = WM * WN, BM = 32 * WI * WM, BN = 32 * WJ * WN;
    static constexpr int SA = (BM + BN) * 128, STAGE = SA + 2 * (BM + BN) * 4;          // rows; two words of scales each
    static constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;                      // loads of a wavefront and stage: 8 rows each
    static constexpr int NS = 2 * (BM + BN) / 64 < WAVES ? 1 : 2 * (BM + BN) / 64 / WAVES, LOADS = LA + LB + NS;     // scales, all
    // results on their way out: 32 rows of 128 bytes (less where a wavefront has fewer) for each wavefront, in the stage that is free
    template <typename T> static constexpr int out_cols() { return 32 * WJ * (int)sizeof(T) < 128 ? 32 * WJ : 128 / (int)sizeof(T); }
    template <typename T> static constexpr int out_row() { return out_cols<T>() * (int)sizeof(T) + 16; }
    static constexpr int OUT = WAVES * 32 * (128 + 16), BIAS = 2 * BN * 4;               // the bias of this tile and of the next
    static constexpr int LDS = BIAS + STAGE + (OUT > STAGE ? OUT : STAGE);
    static_assert(LA >= 1 && LB >= 1, "");
};

__device__ __forceinline__ int spread(int r) { return ((r >> 1) & 7) ^ ((r & 1) << 2); }

template <typename L, typename T> __global__ __launch_bounds__(64 * L::WAVES, L::BM == 256 ? L::WAVES / 4 : 2)
void mxfp4_product_kernel(const ProductArgs P)
{
    constexpr int WI = L::WI, WJ = L::WJ, BM = L::BM, BN = L::BN, STAGE = L::STAGE, LA = L::LA, LB = L::LB, NS = L::NS;
    constexpr int LOADS = L::LOADS, MULS = WI * WJ, READS = WI + WJ, SLOTS = MULS > READS ? MULS : READS;
    extern __shared__ __attribute__((aligned(256))) unsigned char s_tile[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 31, half = lane >> 5;
    const long long row_bytes = (long long)P.nk * 64;

    // Which tiles: the XCDs (every eighth workgroup) get contiguous parts of an order that goes down 4 tiles of C, then right, and
    // their workgroups take turns, so that what an XCD works on at a time is a compact patch and shares its rows in that XCD's L2.
    const int tiles_m = (P.M + BM - 1) / BM, tiles = tiles_m * P.tiles_n, total = tiles * P.split;
    const int xcd = blockIdx.x & 7, part = total >> 3, rest = total & 7, first = xcd * part + min(xcd, rest);
    const int mine = part + (xcd < rest), slots = (gridDim.x + 7 - xcd) >> 3;

    int m0, n0, slice = 0, stages = P.per;
    bool odd = P.nk & 1;                                // the last stage has 128 columns only
    const char *ga, *gb, *gsa, *gsb;
    unsigned off_a[LA], off_b[LB], off_s[NS];           // this lane's part of the loads: 8 rows x 128 bytes each
    auto set_tile = [&](int k) {
        int t = first + k, first_stage = 0;
        if (P.split > 1) {
            slice = __builtin_amdgcn_readfirstlane(t / tiles);
            t -= slice * tiles;
            const int all = (P.nk + 1) >> 1;
            first_stage = slice * P.per;
            stages = min(P.per, all - first_stage);
            odd = (P.nk & 1) && first_stage + stages == all;
        }
        const int group = t / (4 * P.tiles_n), in = t - group * 4 * P.tiles_n, high = min(4, tiles_m - group * 4);
        m0 = __builtin_amdgcn_readfirstlane((group * 4 + in % high) * BM);
        n0 = __builtin_amdgcn_readfirstlane((in / high) * BN);
        ga = reinterpret_cast<const char *>(P.A) + m0 * row_bytes + first_stage * 128LL;
        gb = reinterpret_cast<const char *>(P.B) + n0 * row_bytes + first_stage * 128LL;
        gsa = reinterpret_cast<const char *>(P.SA) + m0 * 4LL + first_stage * 8LL * P.M;
        gsb = reinterpret_cast<const char *>(P.SB) + n0 * 4LL + first_stage * 8LL * P.N;
        int l = lane;
        asm("" : "+v"(l));          // formed here, not kept in registers through the loop over the stages
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const int r = (wave * LA + i) * 8 + (l >> 3);
            off_a[i] = (unsigned)min(r, P.M - 1 - m0) * (unsigned)row_bytes + ((l & 7) ^ spread(r)) * 16;
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const int r = (wave * LB + i) * 8 + (l >> 3);
            off_b[i] = (unsigned)min(r, P.N - 1 - n0) * (unsigned)row_bytes + ((l & 7) ^ spread(r)) * 16;
        }
        // scales: BM + BN words, A's then B's, twice; 64 a load (small tiles: some wavefronts load the same)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            const int at = (wave * NS + i) * 64 % (2 * (BM + BN)) % (BM + BN);
            off_s[i] = 4u * (unsigned)(at < BM ? min(at + l, P.M - 1 - m0) : min(at - BM + l, P.N - 1 - n0));
        }
    };
    const unsigned upper = (((lane >> 2) ^ (lane >> 3)) & 1) << 6;
    // piece g of a stage's loads: LA of A, LB of B, NS of scales.  half_row: the stage has only 64 bytes of a row; the lanes of the
    // other 64 load the first again.
    auto load_piece = [&](int st, int g, bool half_row) {
        unsigned char *to = s_tile + L::BIAS + (st & 1) * STAGE;
        if (g < LA + LB) {
            const bool is_a = g < LA;
            const int i = is_a ? g : g - LA;
            const unsigned off = is_a ? off_a[i] : off_b[i];
            // bit 2 of the lane's piece, (l & 7) ^ spread(row)
            const unsigned behind = (upper ^ (((wave * (is_a ? LA : LB) + i) & 1) << 6)) & (half_row ? 64u : 0u);
            load_to_lds_16((is_a ? ga : gb) + st * 128LL, off - behind,
                           to + (is_a ? 0 : BM * 128) + (wave * (is_a ? LA : LB) + i) * 1024);
        } else {
            const int word = (wave * NS + g - LA - LB) * 64 % (2 * (BM + BN)), second = word >= BM + BN, at = word - second * (BM + BN);
            const long long kc = half_row ? 2 * st : 2 * st + second;
            load_to_lds_4(at < BM ? gsa + kc * 4 * P.M : gsb + kc * 4 * P.N, off_s[g - LA - LB], to + L::SA + word * 4);
        }
    };
    // a tile's first stage, its bias in front (some wavefronts may load the same part)
    auto load_first = [&](int copy) {
        if (P.bias)
            load_to_lds_4(reinterpret_cast<const char *>(P.bias + n0), 4u * (unsigned)min(wave * 64 % BN + lane, P.N - 1 - n0),
                          s_tile + copy * BN * 4 + wave * 64 % BN * 4);
#pragma unroll
        for (int g = 0; g < LOADS; ++g) load_piece(0, g, odd && stages == 1);
    };

    f32x16 acc[WI][WJ];
    const int ra = (wave / L::WN) * 32 * WI, rb = (wave % L::WN) * 32 * WJ;
    const int at = row * 128 + ((half ^ spread(row)) << 4);         // quarter 0; quarter q: piece ^ 2 q
    struct Set { uint4 a[WI], b[WJ]; };
    // fragment g of a quarter, in the order in which the products need them: b 0, a 0, b 1 .., a 1 ..
    auto read_piece = [&](int st, int q, int g, Set &f) {
        const unsigned char *s = s_tile + L::BIAS + (st & 1) * STAGE + (at ^ (q * 32));
        if (g == 1 || g > WJ) {
            const int i = g == 1 ? 0 : g - WJ;
            f.a[i] = *reinterpret_cast<const uint4 *>(s + (ra + 32 * i) * 128);
        } else {
            const int i = g == 0 ? 0 : g - 1;
            f.b[i] = *reinterpret_cast<const uint4 *>(s + (BM + rb + 32 * i) * 128);
        }
    };
    struct Scales { unsigned a[WI], b[WJ]; };
    auto read_scales = [&](int st, int word, Scales &x) {           // word 0: quarters 0 and 1, word 1: 2 and 3
        const unsigned *s = reinterpret_cast<const unsigned *>(s_tile + L::BIAS + (st & 1) * STAGE + L::SA) + word * (BM + BN) + row;
#pragma unroll
        for (int j = 0; j < WJ; ++j) x.b[j] = s[BM + rb + 32 * j];
#pragma unroll
        for (int i = 0; i < WI; ++i) x.a[i] = s[ra + 32 * i];
    };
    auto take_scales = [&](const Scales &x, Scales &y) {            // bytes 0 and 2: this lane's blocks of an even and an odd quarter
#pragma unroll
        for (int i = 0; i < WI; ++i) y.a[i] = x.a[i] >> (8 * half);
#pragma unroll
        for (int j = 0; j < WJ; ++j) y.b[j] = x.b[j] >> (8 * half);
    };
    auto multiply = [&](const Set &f, const Scales &x, int e, auto second) {
        constexpr int SEL = decltype(second)::value ? 2 : 0;
        const int i = e / WJ, j = e % WJ;
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fragment(f.b[j]), fragment(f.a[i]), acc[i][j], 4, 4, SEL,
                                                                    (int)x.b[j], SEL, (int)x.a[i]);
    };

    Set f0, f1;
    Scales x, next;
    using Yes = std::true_type;
    using No = std::false_type;
    // One quarter: the products of f, while fragment e of (st, q) goes to g and a part of a stage's loads is issued (all in the first
    // quarter that may: they have most time then).  Between the fences the written order is kept: left to itself the compiler puts all
    // reads in front and the matrix cores wait for them.
    auto quarter = [&](const Set &f, auto second, Set &g, int st, int q, auto read, auto load, int load_st, bool half_row) {
#pragma unroll
        for (int e = 0; e < SLOTS; ++e) {
            if (decltype(read)::value && e < READS) read_piece(st, q, e, g);
            if (decltype(load)::value)
#pragma unroll
                for (int p = 0; p < LOADS; ++p)
                    if (p * SLOTS / LOADS == e) load_piece(load_st, p, half_row);
            if (e < MULS) multiply(f, x, e, second);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    constexpr int STORES = WI * WJ * 32 * 32 * (int)sizeof(T) / 1024;       // of a wavefront and tile, if nothing of it is cut off
    bool after = false;                                 // that many were issued behind the loads of this tile's first stage
    int k = blockIdx.x >> 3, copy = 0;
    if (k >= mine) return;
    set_tile(k);
    load_first(copy);
    for (; k < mine; k += slots, copy ^= 1) {
#pragma unroll
        for (int i = 0; i < WI; ++i)
#pragma unroll
            for (int j = 0; j < WJ; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        // loads and stores come back in the order in which they were issued: the last tile's stores may still be on their way
        if (after) wait_loads<(STORES < 63 ? STORES : 63)>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read_scales(0, 0, next);
#pragma unroll
        for (int g = 0; g < READS; ++g) read_piece(0, 0, g, f0);
        if (stages > 1)
#pragma unroll
            for (int g = 0; g < LOADS; ++g) load_piece(1, g, odd && stages == 2);
        take_scales(next, x);
        // (the products stand in one straight line for each of the three: in two branches, they would leave the accumulators in
        // different registers, to be copied where the branches meet)
        auto stage = [&](int st, auto load) {
            read_scales(st, 1, next);
            quarter(f0, No(), f1, st, 1, Yes(), No(), 0, false);
            quarter(f1, Yes(), f0, st, 2, Yes(), No(), 0, false);
            take_scales(next, x);
            quarter(f0, No(), f1, st, 3, Yes(), No(), 0, false);
            // the next stage has arrived for every wavefront, and every wavefront has the last quarter of this one
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            read_scales(st + 1, 0, next);
            quarter(f1, Yes(), f0, st + 1, 0, Yes(), load, st + 2, odd && st + 3 == stages);
            take_scales(next, x);
        };
        int st = 0;
        for (; st + 2 < stages; ++st) stage(st, Yes());
        if (st + 1 < stages) stage(st++, No());
        quarter(f0, No(), f1, st, 1, Yes(), No(), 0, false);
        if (!odd) {
            read_scales(st, 1, next);
            quarter(f1, Yes(), f0, st, 2, Yes(), No(), 0, false);
            take_scales(next, x);
            quarter(f0, No(), f1, st, 3, Yes(), No(), 0, false);
        }
        quarter(f1, Yes(), f0, st, 0, No(), No(), 0, false);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                               // every wavefront has the last of its last stage in registers
        asm volatile("" ::: "memory");
        settle(acc);

        const int m_first = m0 + ra, n_first = n0 + rb, n_left = P.N - n_first;
        const bool full = m0 + BM <= P.M && n0 + BN <= P.N;
        T *C_first = static_cast<T *>(P.C) + ((long long)slice * P.M + m_first) * P.ldc + n_first;
        if (k + slots < mine) {                                     // the next tile's first stage comes while this one goes out
            set_tile(k + slots);
            load_first(copy ^ 1);
        }
        after = full;

        // Results: lane holds row m_first + 32 i + l % 32 of C, columns n_first + 32 j + 8 q + 4 (l / 32) .. + 3 in registers 4 q ..
        // 4 q + 3.  Stored from there, an instruction would write 32 pieces of 16 bytes; 32 rows of 128 bytes at a time go through LDS
        // instead (the second stage's place, a part of its own for each wavefront).
        constexpr int COLS = L::template out_cols<T>(), ROW = L::template out_row<T>(), PER16 = 16 / (int)sizeof(T), JS = COLS / 32;
        int l = lane;
        asm("" : "+v"(l));
        unsigned char *s = s_tile + L::BIAS + STAGE + wave * 32 * ROW;
        const float *bias = reinterpret_cast<const float *>(s_tile) + copy * BN + rb;
#pragma unroll
        for (int i = 0; i < WI; ++i)
#pragma unroll
            for (int j0 = 0; j0 < WJ; j0 += JS) {
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
                T *C = C_first + 32LL * i * P.ldc + 32 * j0;
                const int rows = P.M - m_first - 32 * i, cols = n_left - 32 * j0;
                if (full) {
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += AT_ONCE) {
                        const int r = r0 + l / LANES, c = l % LANES;
                        const u32x4 v = *reinterpret_cast<const u32x4 *>(s + r * ROW + c * 16);
                        u32x4_any *to = reinterpret_cast<u32x4_any *>(C + (long long)r * P.ldc + c * PER16);
                        if (BM == 256) __builtin_nontemporal_store(v, to);      // past the operands in L2: 987 -> 946 us at 75,600 x 5120 x 5120
                        else *to = v;
                    }
                } else {
                    const int c = l % LANES * PER16;
                    for (int r = l / LANES; r < 32 && r < rows; r += AT_ONCE) {
                        const unsigned char *from = s + r * ROW + c * (int)sizeof(T);
                        T *to = C + (long long)r * P.ldc + c;
                        if (c + PER16 <= cols) *reinterpret_cast<u32x4_any *>(to) = *reinterpret_cast<const u32x4 *>(from);
                        else
                            for (int e = 0; e < PER16 && c + e < cols; ++e) to[e] = reinterpret_cast<const T *>(from)[e];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);      // else all results leave the accumulators first, for want of registers to memory
            }
    }
}

// C = sum of `split` partial products [M,N], one behind the other, + bias, always in that order.  Bound by reading them, or by its own
// launch: 17 us for 7 parts of 1536 x 1536 (66 MB, 3.9 TB/s), 4 us for 16 of 100 x 200.  grid (ceil(N / 256), rows), block 256
template <typename T> __global__ __launch_bounds__(256) void mxfp4_join_kernel(const float *__restrict__ parts, const ProductArgs P)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= P.N) return;
    const float bias = P.bias ? P.bias[n] : 0.f;
    const size_t part = (size_t)P.M * P.N;
    for (int m = blockIdx.y; m < P.M; m += gridDim.y) {
        const float *p = parts + (size_t)m * P.N + n;
        float v = p[0];
#pragma unroll 4
        for (int s = 1; s < P.split; ++s) v += p[s * part];
        v += bias;
        T *to = static_cast<T *>(P.C) + (long long)m * P.ldc + n;
        if constexpr (sizeof(T) == 4) *to = v;
        else *to = (bf16_t)pack_bf16(v, 0.f);
    }
}

// Few rows (M up to 16): the rows of B are read once, and how fast they come is what counts, so nothing goes through LDS and the
// contraction is split over the wavefronts of a workgroup.  v_mfma_scale_f32_16x16x128_f8f6f4: lane l gives 32 values of row l % 16,
// columns 32 (l / 16) ..: 64 neighbouring bytes of a row, two instructions a cache line.  16 rows of B a workgroup, the rows of A
// behind the last as the last; every wavefront has FEW_PAIRS lines of its rows on their way before it uses the first.  The
// wavefronts' sums meet in LDS and are added in order.
// Measured, this kernel / tiles, us: 5120 x 5120 weights and a row 7.2 / 10.4, 64 x 8192 4.7 / 13.2; the same weights again and again (the
// last cache holds them) and, in brackets, as many sets of weights in turn as come from memory:
//                      1 row                       4 rows                      8 rows                      16 rows
//   15,360 x 5120      10.0 / 12.5 (12.3 / 18.4)   10.2 / 12.4 (13.1 / 18.2)   10.8 / 12.4 (13.6 / 18.2)   12.3 / 12.4 (15.9 / 18.2)
//   20,480 x 5120      12.4 / 12.7 (15.6 / 20.3)   12.3 / 12.8 (16.3 / 20.2)   12.8 / 12.8 (17.2 / 18.8)   14.9 / 12.9 (19.8 / 18.9)
//   20,480 x 8192      17.7 / 18.3 (20.8 / 22.6)   18.2 / 18.4 (21.9 / 21.7)   19.3 / 18.6 (24.0 / 22.0)   22.4 / 19.1 (27.9 / 22.5)
//   32,768 x 8192      26.2 / 21.8 (29.6 / 37.0)   27.1 / 21.5 (31.4 / 34.9)   28.8 / 21.5 (35.3 / 35.0)   33.5 / 21.6 (42.0 / 35.0)
//    4096 x 32,768     14.5 / 16.6 (17.1 / 20.7)   15.0 / 16.8 (18.4 / 20.0)   16.0 / 16.9 (18.9 / 20.1)   19.3 / 17.1 (22.7 / 20.2)
//    4096 x 16,384      8.0 / 11.5 ( 9.4 / 13.4)    8.5 / 11.5 (10.1 / 13.3)    9.2 / 11.7 (10.6 / 13.4)   10.2 / 11.3 (12.3 / 13.6)
//    2048 x 16,384      7.2 /  8.5 ( 8.5 / 11.6)    7.7 /  8.8 ( 9.1 / 10.9)    8.5 /  8.8 ( 9.8 / 11.0)    9.8 /  9.4 (11.7 / 11.6)
//    1024 x 32,768     11.6 /  8.7 (13.0 / 13.0)   12.9 /  8.9 (14.5 / 13.1)   14.3 /  9.0 (16.4 / 13.2)   17.0 /  9.4 (20.4 / 13.4)
//     512 x 65,536     21.3 / 11.1 (23.6 / 18.7)   23.8 / 11.3 (26.4 / 18.7)   26.4 / 11.5 (30.0 / 19.1)   31.7 / 11.6 (37.2 / 19.1)
// so up to 4 rows take it to 10 * 2^24 weights, up to 16 rows to 5 * 2^24; rows longer than 2^14, which one workgroup goes through alone
// here and several workgroups in tiles, only where 4096 of them keep the card busy.  Within the rule 5120 x 13,824 is better in tiles where the
// cache has it: 12.1 / 10.8 (14.1 / 14.0) for one row, 16.3 / 11.6 (19.8 / 13.9) for 16.
// What bounds it: 98 registers, so four wavefronts a SIMD, 512 of the 960 workgroups of 15,360 rows of B at a time, and half of their loads are
// of A.  It reads its 44 MB past L2 at 4.2 TB/s where the last cache has them, at 3.5 TB/s from memory.
constexpr int FEW_ROWS = 16, FEW_PAIRS = 4, FEW_WAVES = 16;
static bool few(int M, int N, int K)
{
    return M <= FEW_ROWS && (long long)N * K <= (M <= 4 ? 10 : 5) << 24 && (K <= 1 << 14 || N >= 4096);
}

template <typename T> __global__ __launch_bounds__(64 * FEW_WAVES) void mxfp4_few_kernel(const ProductArgs P)
{
    __shared__ __attribute__((aligned(16))) float s_sum[FEW_WAVES * 256];          // [wavefront][row of A][row of B]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16, pairs = (P.nk + 1) >> 1;
    const int n = min(n0 + r, P.N - 1), m = min(r, P.M - 1);
    const uint8_t *b = P.B + (long long)n * P.nk * 64 + g * 16, *a = P.A + (long long)m * P.nk * 64 + g * 16;
    const unsigned *sb = reinterpret_cast<const unsigned *>(P.SB) + n, *sa = reinterpret_cast<const unsigned *>(P.SA) + m;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = wave; p0 < pairs; p0 += waves * FEW_PAIRS) {
        constexpr int U = 2 * FEW_PAIRS;
        uint4 vb[U], va[U];
        unsigned xb[U], xa[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kc = 2 * (p0 + (u >> 1) * waves) + (u & 1);
            const bool there = kc < P.nk;                           // zeros behind the end: they add nothing
            vb[u] = there ? *reinterpret_cast<const uint4 *>(b + kc * 64LL) : make_uint4(0, 0, 0, 0);
            xb[u] = there ? sb[(long long)kc * P.N] : 0u;
            va[u] = there ? *reinterpret_cast<const uint4 *>(a + kc * 64LL) : make_uint4(0, 0, 0, 0);
            xa[u] = there ? sa[(long long)kc * P.M] : 0u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(vb[u]), fragment(va[u]), acc, 4, 4, 0, (int)(xb[u] >> (8 * g)), 0,
                                                                   (int)(xa[u] >> (8 * g)));
    }
    asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc));              // (see settle)
    // lane holds row l % 16 of A, rows 4 (l / 16) .. + 3 of B
    *reinterpret_cast<float4 *>(s_sum + (wave * 16 + r) * 16 + 4 * g) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    __syncthreads();
    const int i = threadIdx.x, row = i >> 4, col = n0 + (i & 15);
    if (i >= 256 || row >= P.M || col >= P.N) return;
    float v = 0.f;
    for (int k = 0; k < waves; ++k) v += s_sum[k * 256 + i];
    if (P.bias) v += P.bias[col];
    T *to = static_cast<T *>(P.C) + (long long)row * P.ldc + col;
    if constexpr (sizeof(T) == 4) *to = v;
    else *to = (bf16_t)pack_bf16(v, 0.f);
}

// ---- launchers -------------------------------------------------------------
// slices of a loop so that there are some 2048 workgroups, where the loop has that many steps
static int slices(long long blocks, int steps)
{
    const long long want = (2048 + blocks - 1) / blocks;
    return (int)(want < 1 ? 1 : want > steps ? steps : want);
}

// X goes past the caches from 256 MB on, the size of the last cache level, where its rows are whole lines.  Measured with 75,600 x
// 5120 bf16 values (774 MB) quantise 213 -> 192 us, transposed 291 -> 240, values 212 -> 145 (the codes, 206 MB, then stay cached).
// A smaller X is better left in the caches: 16,384 x 1536 (50 MB), quantise 11.3 us, past them 13.4.  So are rows that share lines:
// 75,599 x 5119, quantise 236 us, past them 262; values 312, past them 419.
static bool streamed(const void *X, int M, int K, int64_t ld, int es)
{
    return (double)M * K * es >= 268435456.0 && (reinterpret_cast<uintptr_t>(X) & 127) == 0 && ld * es % 128 == 0;
}

// f(type, STREAM) with both known at compile time
template <typename F> static int with_types(int dtype, bool stream, F f)
{
    if (dtype == SVG2_BF16) stream ? f((bf16_t *)0, std::true_type()) : f((bf16_t *)0, std::false_type());
    else stream ? f((float *)0, std::true_type()) : f((float *)0, std::false_type());
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int mxfp4_quant_launch(const void *X, int dtype, int M, int G, int Kg, int64_t sm, int64_t sg, bool transposed, void *codes,
                       void *scales, hipStream_t st)
{
    const QuantArgs A = {X, sm, sg, M, G, Kg, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales)};
    const int K = G * Kg, es = dtype == SVG2_BF16 ? 2 : 4;
    const bool lines = G == 1 || (sg * es % 128 == 0 && Kg * es % 128 == 0);
    return with_types(dtype, lines && streamed(X, M, K, sm, es), [&](auto *tp, auto stream) {
        using T = std::remove_pointer_t<decltype(tp)>;
        if (transposed) {
            const int bx = cdiv(cdiv(K, 64), 8) * 8, pairs = cdiv(M, 256), share = (int)((long long)pairs * bx / 2048);
            const int per = 2 * (share < 1 ? 1 : share);
            mxfp4_quant_t_kernel<T, decltype(stream)::value><<<dim3(bx, cdiv(cdiv(M, 128), per)), 256, 0, st>>>(A, per);
        } else {
            const int bx = cdiv(M, 16);
            mxfp4_quant_kernel<T, decltype(stream)::value><<<dim3(bx, slices(bx, cdiv(K, 128))), 256, 0, st>>>(A);
        }
    });
}

int mxfp4_values_launch(const void *codes, const void *scales, int M, int K, int dtype, void *X, int64_t ldx, hipStream_t st)
{
    const uint8_t *c = static_cast<const uint8_t *>(codes), *s = static_cast<const uint8_t *>(scales);
    const int es = dtype == SVG2_BF16 ? 2 : 4;
    return with_types(dtype, streamed(X, M, K, ldx, es), [&](auto *tp, auto stream) {
        using T = std::remove_pointer_t<decltype(tp)>;
        const int bx = cdiv(M, values_rows<T>());
        mxfp4_values_kernel<T, decltype(stream)::value><<<dim3(bx, slices(bx, cdiv(K, 128))), 256, 0, st>>>(c, s, M, K, static_cast<T *>(X), ldx);
    });
}

using Large = Tile<2, 4, 4, 2>;
using Medium = Tile<2, 2, 2, 2>;
using Small = Tile<2, 2, 1, 1>;

template <typename L> static int prepare_tiles()
{
    SVG2_TRY(set_dynamic_lds(reinterpret_cast<const void *>(&mxfp4_product_kernel<L, bf16_t>), L::LDS));
    return set_dynamic_lds(reinterpret_cast<const void *>(&mxfp4_product_kernel<L, float>), L::LDS);
}

int mxfp4_matmul_prepare()
{
    SVG2_TRY(prepare_tiles<Large>());
    SVG2_TRY(prepare_tiles<Medium>());
    return prepare_tiles<Small>();
}

// Microseconds that the product takes with these tiles, by what was measured: `start` a tile, and for each stage of 256 columns
// alone[..] with one workgroup a CU up to full[..] with as many as fit (Large 1, Medium 2, Small 4).  Large tiles do most with
// what they load, small ones leave fewer CUs idle: measured, large / medium / small,
//   8192 x 8192 x 8192    264 / 302 / 459 us        4096 x 5120 x 5120    78 / 65 / 102 us       512 x 5120 x 5120   33 / 17 / 17 us
//   4096 x 4096 x 4096     38 /  45 /  65 us        2048 x 2048 x 2048    18 / 11 /  12 us       300 x 5120 x 5120   40 / 21 / 14 us
template <typename L> static double tile_time(int M, int N, int stages, int split)
{
    constexpr int R = L::BM == 256 ? 1 : L::BM == 128 ? 2 : 4;
    constexpr double start = R == 1 ? 7.0 : R == 2 ? 3.5 : 2.0, alone = R == 1 ? 1.6 : R == 2 ? 0.62 : 0.38, full = R == 1 ? 1.78 : R == 2 ? 1.09 : 0.86;
    const long long tiles = (long long)cdiv(M, L::BM) * cdiv(N, L::BN) * split, rounds = tiles / (256 * R), rest = (tiles - rounds * 256 * R + 255) / 256;
    const double per = cdiv(stages, split);
    const double last = rest == 0 ? 0.0 : start + per * (R == 1 ? alone : alone + (full - alone) * (double)(rest - 1) / (R > 1 ? R - 1 : 1));
    return (double)rounds * (start + per * full) + last;
}

// Which tiles, and in how many parts the contraction: the least time by that model, parts of four stages at least, 16 parts at most (more
// were not measured; 64 x 64 x 1,000,064 runs on 16 workgroups, 126 us, where its operands take 13 to read).  Adding them up is
// a second launch and the parts' way out and back: 5 us, and 0.5 us for each MB of a part.  Measured, one part / as chosen:
//   1536 x 1536 x 75,600   223 / 116 us  (7)        512 x 512 x 65,536    112 /  23 us (16)       64 x 5120 x 13,824    28 / 16 us (3)
//    500 x  700 x 20,000    38 /  17 us  (5)        256 x 256 x 16,384     23 /  14 us (13)      512 x  512 x  8192     13 / 13 us (4)
struct ProductPlan {
    int size, split, per;           // size: 0 small, 1 medium, 2 large
};

static ProductPlan product_plan(int M, int N, int K)
{
    const int stages = cdiv(K, 256);
    ProductPlan best = {0, 1, stages};
    double least = 1e300;
    for (int split = 1; split <= 16 && (split == 1 || stages >= 4 * split); ++split) {
        const int per = cdiv(stages, split);
        if (split > 1 && (cdiv(stages, per) != split || (double)split * M * N > (1 << 28))) continue;
        const double join = split == 1 ? 0.0 : 5.0 + 0.5 * split * (double)M * N * sizeof(float) * 1e-6;
        const double t[3] = {tile_time<Small>(M, N, stages, split), tile_time<Medium>(M, N, stages, split), tile_time<Large>(M, N, stages, split)};
        for (int size = 0; size < 3; ++size)
            if (t[size] + join < least * (size > best.size && split == best.split ? 1.0 : 0.999)) {
                least = t[size] + join;
                best = {size, split, per};
            }
    }
    return best;
}

size_t mxfp4_matmul_ws_bytes(int M, int N, int K)
{
    if (few(M, N, K)) return 256;
    const ProductPlan p = product_plan(M, N, K);
    return p.split == 1 ? 256 : (size_t)p.split * M * N * sizeof(float);
}

template <typename L, typename T> static int product_tiles(ProductArgs P, hipStream_t st)
{
    P.tiles_n = cdiv(P.N, L::BN);
    const int tiles = cdiv(P.M, L::BM) * P.tiles_n * P.split, resident = 256 * (L::BM == 256 ? 1 : L::BM == 128 ? 2 : 4);
    mxfp4_product_kernel<L, T><<<tiles < resident ? tiles : resident, 64 * L::WAVES, L::LDS, st>>>(P);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

template <typename T> static int product_sized(int size, const ProductArgs &P, hipStream_t st)
{
    return size == 2 ? product_tiles<Large, T>(P, st) : size == 1 ? product_tiles<Medium, T>(P, st) : product_tiles<Small, T>(P, st);
}

static int product_few(const ProductArgs &P, int out_dtype, hipStream_t st)
{
    // 4 wavefronts, 8 or 16: enough of them for the whole card and for every line of a row to be on its way at once, not more than
    // there are lines in a row
    const int blocks = cdiv(P.N, 16), pairs = cdiv(P.nk, 2);
    int waves = 4;
    while (waves < FEW_WAVES && waves < pairs && ((long long)blocks * waves < 4096 || waves * FEW_PAIRS < pairs)) waves *= 2;
    if (out_dtype == SVG2_BF16) mxfp4_few_kernel<bf16_t><<<blocks, 64 * waves, 0, st>>>(P);
    else mxfp4_few_kernel<float><<<blocks, 64 * waves, 0, st>>>(P);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int mxfp4_matmul_launch(const void *A, const void *SA, const void *B, const void *SB, int M, int N, int K, const float *bias,
                        int out_dtype, void *C, int64_t ldc, void *ws, hipStream_t st)
{
    ProductArgs P = {static_cast<const uint8_t *>(A), static_cast<const uint8_t *>(B), static_cast<const uint8_t *>(SA),
                     static_cast<const uint8_t *>(SB), M, N, cdiv(K, 128), bias, C, ldc, 0, 1, cdiv(K, 256)};
    if (few(M, N, K)) return product_few(P, out_dtype, st);
    const ProductPlan p = product_plan(M, N, K);
    if (p.split == 1) return out_dtype == SVG2_BF16 ? product_sized<bf16_t>(p.size, P, st) : product_sized<float>(p.size, P, st);
    P.split = p.split;
    P.per = p.per;
    ProductArgs parts = P;
    parts.bias = nullptr;
    parts.C = ws;
    parts.ldc = N;
    SVG2_TRY(product_sized<float>(p.size, parts, st));
    const dim3 grid(cdiv(N, 256), M < 4096 ? M : 4096);
    if (out_dtype == SVG2_BF16) mxfp4_join_kernel<bf16_t><<<grid, 256, 0, st>>>(static_cast<const float *>(ws), P);
    else mxfp4_join_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float *>(ws), P);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

}  // namespace svg2

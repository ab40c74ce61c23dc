// 8-bit floating point (E4M3) operands with a scale for each block of 128: quantisation, the values back, and the product
// C = A B^T + bias.  Storage and scales: svg2_fp8_blocks.h.
//
// The scales are powers of two, so that the matrix cores multiply by them (v_mfma_scale_*) and a product needs no instruction of its own
// for them; what a power of two costs against any number is at most one of E4M3's 15 binades, no bit of a normal number.
#include <type_traits>

#include "svg2_fp8_blocks.h"

namespace svg2 {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// f(0), f(1), .. with each number known at compile time
template <int FROM, int TO, typename F> __device__ __forceinline__ void static_for(F f)
{
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>());
        static_for<FROM + 1, TO>(f);
    }
}

struct BlockQuantArgs {
    const void *X;
    long long sm, sg;               // strides of rows and of groups of columns
    int M, G, Kg;                   // X is [M, G, Kg]; K = G Kg columns
    uint8_t *codes, *scales;        // operand of M rows and K columns
    uint8_t *codes_t, *scales_t;    // operand of K rows and M columns
    int per_xcd;                    // tiles that follow each other on one XCD; 0: every eighth
};

template <typename T> __device__ __forceinline__ const T *element(const BlockQuantArgs &A, long long m, int k)
{
    const int g = A.G == 1 ? 0 : k / A.Kg;
    return static_cast<const T *>(A.X) + m * A.sm + g * A.sg + (k - g * A.Kg);
}

// eight neighbouring columns: one load where they are all there and in one group, whatever their address; zeros behind K
template <typename T, bool STREAM> __device__ __forceinline__ Raw<T> load_columns(const BlockQuantArgs &A, long long m, int k, int K)
{
    if (k + 8 <= K && (A.G == 1 || k % A.Kg + 8 <= A.Kg)) return load_raw<T, STREAM>(element<T>(A, m, k));
    return raw_of<T>([&](int i) { return k + i < K ? *element<T>(A, m, k + i) : (T)0; });
}

// rows: grid (ceil(M / 16), slices of the columns), block 256: 16 lanes a block of 128 columns, whose eight values each stay in
// registers; the block's maximum goes round the 16 lanes without LDS.  Bound by HBM: 16,384 x 5120 bf16 46 us, 5.4 TB/s, 75,600 x 5120 235, 4.9.
template <typename T, bool STREAM> __global__ __launch_bounds__(256) void fp8_blocks_rows_kernel(const BlockQuantArgs A)
{
    const int lane16 = threadIdx.x & 15, K = A.G * A.Kg, nk = (K + 127) / 128, all = (nk + 3) & ~3;
    const long long m = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (m >= A.M) return;                       // whole groups of 16 lanes
    for (int kc = blockIdx.y; kc < all; kc += gridDim.y) {
        unsigned byte = 0;
        if (kc < nk) {
            float v[8], inv;
            decode<T>(load_columns<T, STREAM>(A, m, kc * 128 + lane16 * 8, K), v);
            byte = e4m3_block_scale(max16(largest8(v)), inv);
            *reinterpret_cast<uint2 *>(A.codes + m * (nk * 128LL) + kc * 128 + lane16 * 8) = e4m3_codes8(v, inv);
        }
        if (lane16 == 0) A.scales[((long long)(kc >> 2) * A.M + m) * 4 + (kc & 3)] = (uint8_t)byte;
    }
}

// tiles of 128 x 128 for the transposed operand, for both from one read, and for square blocks.
// grid: workgroups stride over the tiles, those of one row of tiles neighbours, on one XCD where they share lines; block 256: a thread holds 8 rows x 8 columns, as they are in
// memory.  The maximum of a row goes round 16 lanes, that of a column over the wavefront's four groups of rows and, through LDS, the four
// wavefronts.  The codes of eight rows of a column are eight bytes: they go through LDS, column by column, and leave as lines of 128 bytes.
// Bound by HBM: 16,384 x 5120 bf16 both ways 67 us, 5.0 TB/s (rows and transposed in calls of their own 94), transposed 48, in squares both ways 61;
// small ones by their few workgroups (16,384 x 1536 both ways 25 us, 1536 of them).  Rows that are not whole lines (75,599 x 5119 both ways 356 us,
// 31,299 x 2047 65) have neighbouring tiles read the same ones, twice from memory if those go to the next XCD each (415, 107).
template <typename T, bool STREAM, bool ROWS, bool COLS, bool SQUARE> __global__ __launch_bounds__(256) void fp8_blocks_tile_kernel(const BlockQuantArgs A)
{
    __shared__ unsigned s_top[4][128];
    __shared__ __attribute__((aligned(16))) uint8_t s_codes[COLS ? 128 * 144 : 16];     // a column's 128 codes and 16 bytes: stores of 8 bytes spread over the banks
    const int K = A.G * A.Kg, nk = (K + 127) / 128, nm = (A.M + 127) / 128;
    const int lane16 = threadIdx.x & 15, rows8 = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const long long all = (long long)nm * nk, turns = A.per_xcd ? 8LL * A.per_xcd : all;
    for (long long turn = blockIdx.x; turn < turns; turn += gridDim.x) {
        const long long tile = A.per_xcd ? (turn & 7) * A.per_xcd + (turn >> 3) : turn;
        if (tile >= all) continue;
        const int kc = (int)(tile % nk), mc = (int)(tile / nk), k0 = kc * 128 + lane16 * 8;
        const long long m0 = (long long)mc * 128 + rows8 * 8;
        Raw<T> x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (m0 + i < A.M) x[i] = load_columns<T, STREAM>(A, m0 + i, k0, K);
            else x[i] = raw_of<T>([](int) { return (T)0; });
        }
        auto row_result = [&](int i, const float *v, unsigned top) {
            float inv;
            const unsigned byte = e4m3_block_scale(top, inv);
            const uint2 c = e4m3_codes8(v, inv);
            if (m0 + i < A.M) {
                *reinterpret_cast<uint2 *>(A.codes + (m0 + i) * (nk * 128LL) + kc * 128 + lane16 * 8) = c;
                uint8_t *s = A.scales + ((long long)(kc >> 2) * A.M + m0 + i) * 4;
                if (lane16 == 0) s[kc & 3] = (uint8_t)byte;
                if (kc == nk - 1 && lane16 > (kc & 3) && lane16 < 4) s[lane16] = 0;
            }
        };
        unsigned col_top[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) col_top[e] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v[8];
            decode<T>(x[i], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) col_top[e] = max(col_top[e], mag(v[e]));
            if (ROWS && !SQUARE) row_result(i, v, max16(largest8(v)));
            // one row after another, and its values formed again below: kept, the 64 of them and what they become take 213 registers
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (unsigned w = 0; w < sizeof(T) / 2; ++w) asm volatile("" : "+v"(x[i].q[w]));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            col_top[e] = max(col_top[e], (unsigned)__shfl_xor((int)col_top[e], 16));
            col_top[e] = max(col_top[e], (unsigned)__shfl_xor((int)col_top[e], 32));
            if ((threadIdx.x & 63) < 16) s_top[wave][lane16 * 8 + e] = col_top[e];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = lane16 * 8 + e;
            col_top[e] = max(max(s_top[0][k], s_top[1][k]), max(s_top[2][k], s_top[3][k]));
        }
        if (SQUARE) {
            unsigned all = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) all = max(all, col_top[e]);
            all = max16(all);
#pragma unroll
            for (int e = 0; e < 8; ++e) col_top[e] = all;
            if (ROWS)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float v[8];
                    decode<T>(x[i], v);
                    row_result(i, v, all);
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
        if (COLS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float inv, v[8];
                const unsigned byte = e4m3_block_scale(col_top[e], inv);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = value<T>(x[i], e);
                *reinterpret_cast<uint2 *>(s_codes + (lane16 * 8 + e) * 144 + rows8 * 8) = e4m3_codes8(v, inv);
                const long long r = k0 + e;
                if (r < K && rows8 < 4) {
                    uint8_t *s = A.scales_t + ((long long)(mc >> 2) * K + r) * 4;
                    if (rows8 == (mc & 3)) s[rows8] = (uint8_t)byte;
                    else if (mc == nm - 1 && rows8 > (mc & 3)) s[rows8] = 0;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            __syncthreads();
            for (int p = threadIdx.x; p < 128 * 8; p += 256) {
                const long long r = (long long)kc * 128 + (p >> 3);
                if (r < K)
                    *reinterpret_cast<u32x4 *>(A.codes_t + r * (nm * 128LL) + mc * 128 + (p & 7) * 16) =
                        *reinterpret_cast<const u32x4 *>(s_codes + (p >> 3) * 144 + (p & 7) * 16);
            }
        }
        __syncthreads();                        // s_top and s_codes have been read
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

// grid (ceil(M / 16), slices of the columns), block 256: 16 lanes a block, eight codes each.  Bound by the writes: 16,384 x 5120 bf16 39 us, the codes
// from the last cache; 75,600 x 5120 237, 4.9 TB/s
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void fp8_blocks_values_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                                int M, int K, T *__restrict__ X, long long ldx)
{
    const int lane16 = threadIdx.x & 15, nk = (K + 127) / 128;
    const long long m = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (m >= M) return;
    for (int kc = blockIdx.y; kc < nk; kc += gridDim.y) {
        const uint2 c = *reinterpret_cast<const uint2 *>(codes + m * (nk * 128LL) + kc * 128 + lane16 * 8);
        float a, b, v[8];
        scale_factors(scales[((long long)(kc >> 2) * M + m) * 4 + (kc & 3)], a, b);
        const f32x2 p[4] = {__builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)c.x, true),
                            __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)c.y, true)};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[i >> 1][i & 1] * a * b;
        const int k = kc * 128 + lane16 * 8;
        T *x = X + m * ldx + k;
        if (k + 8 <= K) store8<T, STREAM>(x, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < K) store_one(x + i, v[i]);
    }
}

// ---- the product -----------------------------------------------------------
struct BlockProductArgs {
    const uint8_t *A, *B, *SA, *SB; // codes [M, Kp], [N, Kp]; scales [ceil(Kp/512), M, 4], [ceil(Kp/512), N, 4]
    int M, N, nk;                   // nk = Kp / 128
    int rows_a;                     // of A's scales: M, or more where these are some rows of a larger product
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

// Wait states between the last matrix instructions and the vector instructions that read their results, more than either the compiler
// or the hardware asks for.  The results are operands of the statement, all of them of one: it stands behind every instruction that writes
// them and before every one that reads them, which an s_nop by itself does not.
template <int I, int J> __device__ __forceinline__ void settle(f32x16 (&a)[I][J])
{
    static_assert(I * J == 8 || I * J == 4 || I * J == 1, "");
    if constexpr (I * J == 8)
        asm volatile("s_nop 15\n\ts_nop 15" : "+v"(a[0][0]), "+v"(a[0][1]), "+v"(a[1][0]), "+v"(a[1][1]), "+v"(a[2][0]), "+v"(a[2][1]),
                     "+v"(a[3][0]), "+v"(a[3][1]));
    else if constexpr (I * J == 4) asm volatile("s_nop 15\n\ts_nop 15" : "+v"(a[0][0]), "+v"(a[0][1]), "+v"(a[1][0]), "+v"(a[1][1]));
    else asm volatile("s_nop 15\n\ts_nop 15" : "+v"(a[0][0]));
}

// How exact the matrix cores are on E4M3 (measured; the same for every instruction that takes it): products of eight neighbouring columns
// are added with 13 bits below the power of two of the largest of them, what is below is cut off; sums of such groups have fp32's 24
// bits.  That is 1.4e-5 of a sum of 64 Gaussian products (rms), against 5e-9 for the same numbers as bf16, and against the 2^-8 by which a bf16
// result may be rounded; where large products cancel it is more of the result, up to 7 * 2^-13 of the sum of each eight's largest.  So a bf16 result is formed by them, at twice the rate, and an fp32 result (EXACT) from the values as bf16, which has them all.
struct Converted { bf16x8 q[4]; };                      // 32 values

__device__ __forceinline__ Converted convert(const i32x8 &f, unsigned byte)
{
    Converted c;
    const float scale = __uint_as_float(byte << 23);
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)f[w], scale, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)f[w], scale, true);
        c.q[w >> 1][4 * (w & 1)] = lo[0];
        c.q[w >> 1][4 * (w & 1) + 1] = lo[1];
        c.q[w >> 1][4 * (w & 1) + 2] = hi[0];
        c.q[w >> 1][4 * (w & 1) + 3] = hi[1];
    }
    return c;
}

// The tiled product.  v_mfma_scale_f32_32x32x64_f8f6f4 on E4M3 operands: lane l gives 32 values of row l % 32 and their scale; which 32 of the
// 64 columns is the same for both operands, and they all have one scale, so their order does not matter.  The rows of B go in
// first: a lane's results are then neighbours in a row of C.
//
// Workgroup: WM x WN wavefronts of 32 WI x 32 WJ results, one tile of C after another.  A stage is a block, 128 columns of the tile's rows of either
// side: a cache line of each.  Two stages are in LDS, one on its way while the other is used, straight from memory (global_load_lds).
// A stage is used in slots, one for each of two halves of the columns and 32 rows of A: WJ products each.  The rows of A are read from LDS AHEAD
// slots before they are used, those of B half a stage before.  The one barrier of a stage stands where its last reads have been made:
// the next stage has arrived by then, and this one's place is free.  The scales of four stages are a word of a row, which comes with each of the
// four: a branch around it would cut the loop in two, and the compiler moves products over such a cut.
// Where there are few tiles and many stages, a part of the stages is a tile of its own (split), and fp8_blocks_join_kernel adds them up.
// In LDS row r has 128 bytes, its 16-byte piece c at c ^ spread(r): eight neighbouring rows then take every bank once.
// Rows behind the last are read as the last and not stored.
// What bounds it is the power: a loop of nothing but this instruction on operands in registers does 3.7 PFLOP/s (operands of zeros 5.0), its clock
// at 1.8 GHz of 2.4.  8192 x 8192 x 8192, 400 us, 2.75 PFLOP/s: the matrix pipes are busy 70 % of the cycles, at 1.8 GHz too, since operands on
// their way through LDS take power as well; 75,600 x 5120 x 5120, 1560 us, 2.54 PFLOP/s, 69 %: a tile's results take some 5 us beyond its 40
// stages.  fp32 results: 16,384 x 5120 x 5120 600 us, 1.43 PFLOP/s, busy 77 % at 1.69 GHz.
// Four stages in LDS for small tiles, three on their way, change nothing (1021 x 1537 x 1000 6.9 us either way).
// Steps, 8192 x 8192 x 8192: two stages in LDS, scales every fourth stage 415 us (the branch around them had every product of a stage moved behind its
// barrier); scales every stage, no branch 408; loads behind a product each 400.
template <int WM_, int WN_, int WI_, int WJ_> struct Tile {
    static constexpr int WM = WM_, WN = WN_, WI = WI_, WJ = WJ_, WAVES = WM * WN, BM = 32 * WI * WM, BN = 32 * WJ * WN;
    static constexpr int STAGE = (BM + BN) * 128;
    static constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES, LOADS = LA + LB;     // loads of a wavefront and stage: 8 rows each
    static constexpr int NS = (BM + BN) / 64 < WAVES ? 1 : (BM + BN) / 64 / WAVES;      // and of scales
    static constexpr int SLOTS = 2 * WI, AHEAD = WI == 4 ? 3 : WI, RING = AHEAD < 2 ? 2 : 4;
    // results on their way out: 32 rows of 128 bytes (less where a wavefront has fewer) for each wavefront, in the stage that is free
    template <typename T> static constexpr int out_cols() { return 32 * WJ * (int)sizeof(T) < 128 ? 32 * WJ : 128 / (int)sizeof(T); }
    template <typename T> static constexpr int out_row() { return out_cols<T>() * (int)sizeof(T) + 16; }
    static constexpr int OUT = WAVES * 32 * (128 + 16), BIAS = 2 * BN * 4;               // the bias of this tile and of the next
    static constexpr int SCALES = 2 * (BM + BN) * 4, FRONT = BIAS + SCALES;              // a word of every row, of these four stages and the next
    static constexpr int LDS = FRONT + STAGE + (OUT > STAGE ? OUT : STAGE);
    static_assert(LA >= 1 && LB >= 1 && SLOTS % RING == 0, "");
};

__device__ __forceinline__ int spread(int r) { return ((r >> 1) & 7) ^ ((r & 1) << 2); }

template <typename L, typename T, bool EXACT> __global__ __launch_bounds__(64 * L::WAVES, L::BM == 256 ? L::WAVES / 4 : 2)
void fp8_blocks_product_kernel(const BlockProductArgs P)
{
    constexpr int WI = L::WI, WJ = L::WJ, BM = L::BM, BN = L::BN, STAGE = L::STAGE, LA = L::LA, LB = L::LB;
    constexpr int LOADS = L::LOADS, SLOTS = L::SLOTS, AHEAD = L::AHEAD, RING = L::RING, BARRIER = SLOTS - AHEAD;
    extern __shared__ __attribute__((aligned(256))) unsigned char s_tile[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 31, half = lane >> 5;
    const long long row_bytes = (long long)P.nk * 128;

    // Which tiles: the XCDs (every eighth workgroup) get contiguous parts of an order that goes down 4 tiles of C, then right, and
    // their workgroups take turns, so that what an XCD works on at a time is a compact patch and shares its rows in that XCD's L2.
    const int tiles_m = (P.M + BM - 1) / BM, tiles = tiles_m * P.tiles_n, total = tiles * P.split;
    const int xcd = blockIdx.x & 7, part = total >> 3, rest = total & 7, first = xcd * part + min(xcd, rest);
    const int mine = part + (xcd < rest), slots = (gridDim.x + 7 - xcd) >> 3;
    const int ra = (wave / L::WN) * 32 * WI, rb = (wave % L::WN) * 32 * WJ;

    int m0, n0, slice = 0, stages = P.per, first_stage = 0;
    const char *ga, *gb;
    unsigned off_a[LA], off_b[LB];                      // this lane's part of the loads: 8 rows x 128 bytes each
    unsigned off_s[L::NS];
    unsigned wa[WI], wb[WJ], next_a[WI], next_b[WJ];    // scales of the rows that this lane gives, this stage's in the lowest byte
    auto set_tile = [&](int k) {
        int t = first + k;
        if (P.split > 1) {
            slice = __builtin_amdgcn_readfirstlane(t / tiles);
            t -= slice * tiles;
            first_stage = slice * P.per;
            stages = min(P.per, P.nk - first_stage);
        }
        const int group = t / (4 * P.tiles_n), in = t - group * 4 * P.tiles_n, high = min(4, tiles_m - group * 4);
        m0 = __builtin_amdgcn_readfirstlane((group * 4 + in % high) * BM);
        n0 = __builtin_amdgcn_readfirstlane((in / high) * BN);
        ga = reinterpret_cast<const char *>(P.A) + m0 * row_bytes + first_stage * 128LL;
        gb = reinterpret_cast<const char *>(P.B) + n0 * row_bytes + first_stage * 128LL;
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
        // scales: BM + BN words, A's then B's, 64 a load (small tiles: some wavefronts load the same)
#pragma unroll
        for (int i = 0; i < L::NS; ++i) {
            const int word = (wave * L::NS + i) * 64 % (BM + BN);
            off_s[i] = 4u * (unsigned)(word < BM ? min(word + l, P.M - 1 - m0) : min(word - BM + l, P.N - 1 - n0));
        }
    };
    // piece g of a stage's loads: LA of A, LB of B
    auto load_piece = [&](int st, int g) {
        unsigned char *to = s_tile + L::FRONT + (st & 1) * STAGE;
        if (g < LA) load_to_lds_16(ga + st * 128LL, off_a[g], to + (wave * LA + g) * 1024);
        else load_to_lds_16(gb + st * 128LL, off_b[g - LA], to + BM * 128 + (wave * LB + g - LA) * 1024);
    };
    auto load_scales = [&](int st) {                    // of stages st .. st + 3
        const long long w = (first_stage + st) >> 2;
#pragma unroll
        for (int i = 0; i < L::NS; ++i) {
            const int word = (wave * L::NS + i) * 64 % (BM + BN);
            load_to_lds_4(reinterpret_cast<const char *>(word < BM ? P.SA + 4 * (w * P.rows_a + m0) : P.SB + 4 * (w * P.N + n0)), off_s[i],
                          s_tile + L::BIAS + ((st >> 2) & 1) * (BM + BN) * 4 + word * 4);
        }
    };
    // a tile's first stage, its bias in front (some wavefronts may load the same part)
    auto load_first = [&](int copy) {
        if (P.bias)
            load_to_lds_4(reinterpret_cast<const char *>(P.bias + n0), 4u * (unsigned)min(wave * 64 % BN + lane, P.N - 1 - n0),
                          s_tile + copy * BN * 4 + wave * 64 % BN * 4);
        load_scales(0);
#pragma unroll
        for (int g = 0; g < LOADS; ++g) load_piece(0, g);
    };

    f32x16 acc[WI][WJ];
    const int at = row * 128 + ((half ^ spread(row)) << 4);         // piece 0 of the first half of a stage; piece p of half h: ^ (64 h + 32 p)
    i32x8 a[RING], b[2][WJ];
    Converted cb[EXACT ? WJ : 1];
    auto read = [&](int st, int h, int rows) {
        const unsigned char *s = s_tile + L::FRONT + (st & 1) * STAGE + rows * 128;
        const uint4 x = *reinterpret_cast<const uint4 *>(s + (at ^ (64 * h))), y = *reinterpret_cast<const uint4 *>(s + (at ^ (64 * h + 32)));
        return i32x8{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
    };
    auto read_scales = [&](int st, unsigned *xa, unsigned *xb) {
        const unsigned *s = reinterpret_cast<const unsigned *>(s_tile + L::BIAS) + ((st >> 2) & 1) * (BM + BN) + row;
#pragma unroll
        for (int i = 0; i < WI; ++i) xa[i] = s[ra + 32 * i];
#pragma unroll
        for (int j = 0; j < WJ; ++j) xb[j] = s[BM + rb + 32 * j];
    };
    auto take_scales = [&](int st) {
        const int shift = 8 * (st & 3);
#pragma unroll
        for (int i = 0; i < WI; ++i) wa[i] = next_a[i] >> shift;
#pragma unroll
        for (int j = 0; j < WJ; ++j) wb[j] = next_b[j] >> shift;
    };
    // Slot e: the reads that fall into it (from the next stage where there is one: `next`), its products, and its share of the loads of the stage
    // behind that (`load`).  In one piece behind the barrier, the 64 loads of a workgroup keep its wavefronts from the matrix cores for as long
    // as the memory pipe takes to accept them, some 17 cycles each: 8192 x 8192 x 8192 423 us, behind a product each 400.
    auto slot = [&](int st, auto slot_number, auto next, auto load) {
        constexpr int e = decltype(slot_number)::value, h = e / WI, i = e % WI, to = e + AHEAD;
        constexpr bool more = decltype(next)::value;
        if (to < SLOTS) a[to % RING] = read(st, to / WI, ra + 32 * (to % WI));
        else if (more) a[to % RING] = read(st + 1, 0, ra + 32 * (to - SLOTS));
        // B of the second half in the first slots, of the next stage's first half behind the barrier
#pragma unroll
        for (int j = 0; j < WJ; ++j) {
            if (h == 0 && j * WI / WJ == i) b[1][j] = read(st, 1, BM + rb + 32 * j);
            if (more && e >= BARRIER && min(j, AHEAD - 1) == e - BARRIER) b[0][j] = read(st + 1, 0, BM + rb + 32 * j);
        }
        auto loads = [&](int j) {
            constexpr int PLACES = AHEAD * WJ;
            if (decltype(load)::value && e >= BARRIER) {
                if (e == BARRIER && j == 0) load_scales(st + 2);
#pragma unroll
                for (int g = 0; g < LOADS; ++g)
                    if (g * PLACES / LOADS == (e - BARRIER) * WJ + j) load_piece(st + 2, g);
            }
        };
        if constexpr (EXACT) {
            if (i == 0)
#pragma unroll
                for (int j = 0; j < WJ; ++j) cb[j] = convert(b[h][j], wb[j] & 255u);
            const Converted ca = convert(a[e % RING], wa[i] & 255u);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < WJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cb[j].q[q], ca.q[q], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < WJ; ++j) loads(j);
        } else {
#pragma unroll
            for (int j = 0; j < WJ; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[h][j], a[e % RING], acc[i][j], 0, 0, 0, (int)wb[j], 0, (int)wa[i]);
                __builtin_amdgcn_sched_barrier(0);
                loads(j);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // One stage: a straight line of products, of which there are three (in branches the accumulators would be left in different registers,
    // to be copied where the branches meet).  load: there is a stage behind the next.
    auto stage = [&](int st, auto next, auto load) {
        constexpr bool more = decltype(next)::value;
        static_for<0, BARRIER>([&](auto e) { slot(st, e, next, load); });
        // the next stage has arrived for every wavefront, and every wavefront has the last of this one in registers
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (more) read_scales(st + 1, next_a, next_b);
        static_for<BARRIER, SLOTS>([&](auto e) { slot(st, e, next, load); });
        if (more) take_scales(st + 1);
    };
    using Yes = std::true_type;
    using No = std::false_type;

    constexpr int STORES = WI * WJ * 32 * 32 * (int)sizeof(T) / 1024;       // of a wavefront and tile, if nothing of it is cut off
    bool after = false;                                 // that many were issued behind the loads of this tile's first stage
    int k = blockIdx.x >> 3, copy = 0;
    if (k >= mine) return;
    set_tile(k);
    load_first(copy);
    // the second stage of the first tile comes with the first; later tiles' second stages have to wait for the results that leave through their place
    auto load_second = [&]() {
        if (stages > 1)
#pragma unroll
            for (int g = 0; g < LOADS; ++g) load_piece(1, g);
    };
    load_second();
    bool second = true;
    for (; k < mine; k += slots, copy ^= 1) {
#pragma unroll
        for (int i = 0; i < WI; ++i)
#pragma unroll
            for (int j = 0; j < WJ; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        // loads and stores come back in the order in which they were issued: the last tile's stores may still be on their way
        if (after) wait_loads<(STORES < 63 ? STORES : 63)>();
        else if (second && stages > 1) wait_loads<LOADS>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read_scales(0, next_a, next_b);
        take_scales(0);
#pragma unroll
        for (int j = 0; j < WJ; ++j) b[0][j] = read(0, 0, BM + rb + 32 * j);
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) a[e % RING] = read(0, e / WI, ra + 32 * (e % WI));
        if (!second) load_second();
        second = false;
        int st = 0;
        for (; st + 2 < stages; ++st) stage(st, Yes(), Yes());
        if (st + 1 < stages) stage(st++, Yes(), No());
        stage(st, No(), No());
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
        unsigned char *s = s_tile + L::FRONT + STAGE + wave * 32 * ROW;
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
                        if (BM == 256) __builtin_nontemporal_store(v, to);      // past the operands in L2 (75,600 x 1536 x 1536 181 -> 164 us)
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

// C = sum of `split` partial products [M,N], one behind the other, + bias, always in that order; a thread takes four columns where N is a multiple
// of four.  grid (ceil(N / (256 * PER)), rows), block 256
template <typename T, int PER> __global__ __launch_bounds__(256) void fp8_blocks_join_kernel(const float *__restrict__ parts, const BlockProductArgs P)
{
    typedef float vec __attribute__((ext_vector_type(PER)));
    const int n = (blockIdx.x * 256 + threadIdx.x) * PER;
    if (n >= P.N) return;
    vec bias;
#pragma unroll
    for (int e = 0; e < PER; ++e) bias[e] = P.bias ? P.bias[n + e] : 0.f;
    const size_t part = (size_t)P.M * P.N;
    for (int m = blockIdx.y; m < P.M; m += gridDim.y) {
        const float *p = parts + (size_t)m * P.N + n;
        vec v = *reinterpret_cast<const vec *>(p);
#pragma unroll 4
        for (int s = 1; s < P.split; ++s) v += *reinterpret_cast<const vec *>(p + s * part);
        v += bias;
        T *to = static_cast<T *>(P.C) + (long long)m * P.ldc + n;
#pragma unroll
        for (int e = 0; e < PER; ++e) store_one(to + e, v[e]);
    }
}

// Few rows (M up to 16): the rows of B are read once, and how fast they come is what counts, so nothing goes through LDS and the
// contraction is split over the wavefronts of a workgroup.  16 rows of B a workgroup, the rows of A behind the last as the last; a lane gives 32
// neighbouring bytes of row l % 16, four lanes the block of 128.  Every wavefront has FEW_BLOCKS blocks of its rows on their way before it
// uses the first (four 15.6 us at 15,360 x 5120 weights, eight, whose registers go to memory, 116).  The wavefronts' sums meet in LDS and are
// added in order.
// Measured, this kernel / tiles, us; the same weights again and again (the last cache holds them) and, in brackets, as many sets of weights in
// turn as come from memory:
//                     1 row                       8 rows                      16 rows
//   15,360 x 5120     15.1 / 18.7 (16.8 / 21.0)   18.4 / 19.2 (20.6 / 21.9)   21.7 / 19.9 (24.7 / 23.1)
//    5120 x 5120       8.4 / 11.3 ( 9.5 / 11.7)   10.1 / 11.5 (11.1 / 12.0)   11.8 / 11.5 (13.2 / 12.1)
//   20,480 x 8192     29.7 / 29.7 (33.2 / 35.8)   35.2 / 30.1 (40.2 / 36.4)   41.2 / 30.9 (47.1 / 37.2)
//    4096 x 16,384    16.0 / 15.5 (17.0 / 18.8)   18.3 / 16.0 (18.5 / 19.2)   19.7 / 16.2 (20.2 / 19.4)
//    2048 x 16,384    12.0 / 11.4 (13.3 / 13.1)   15.1 / 11.8 (16.1 / 13.5)   17.6 / 11.5 (18.5 / 13.8)
// so up to 4 rows take it to 10 * 2^24 weights, up to 8 rows to 5 * 2^24, of rows up to 8192 long.
constexpr int FEW_BLOCKS = 2, FEW_WAVES = 16;

template <typename T, bool EXACT> __global__ __launch_bounds__(64 * FEW_WAVES) void fp8_blocks_few_kernel(const BlockProductArgs P)
{
    __shared__ __attribute__((aligned(16))) float s_sum[FEW_WAVES * 256];          // [wavefront][row of A][row of B]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16;
    const int n = min(n0 + r, P.N - 1), m = min(r, P.M - 1);
    const uint8_t *b = P.B + (long long)n * P.nk * 128 + g * 32, *a = P.A + (long long)m * P.nk * 128 + g * 32;
    const uint8_t *sb = P.SB + n * 4LL, *sa = P.SA + m * 4LL;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const i32x8 none = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k0 = wave; k0 < P.nk; k0 += waves * FEW_BLOCKS) {
        i32x8 vb[FEW_BLOCKS], va[FEW_BLOCKS];
        unsigned xb[FEW_BLOCKS], xa[FEW_BLOCKS];
#pragma unroll
        for (int u = 0; u < FEW_BLOCKS; ++u) {
            const int kc = k0 + u * waves;
            const bool there = kc < P.nk;                           // zeros behind the end: they add nothing
            vb[u] = there ? *reinterpret_cast<const i32x8 *>(b + kc * 128LL) : none;
            xb[u] = there ? sb[(long long)(kc >> 2) * P.N * 4 + (kc & 3)] : 0u;
            va[u] = there ? *reinterpret_cast<const i32x8 *>(a + kc * 128LL) : none;
            xa[u] = there ? sa[(long long)(kc >> 2) * P.rows_a * 4 + (kc & 3)] : 0u;
        }
#pragma unroll
        for (int u = 0; u < FEW_BLOCKS; ++u) {
            if constexpr (EXACT) {
                const Converted cb = convert(vb[u], xb[u]), ca = convert(va[u], xa[u]);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cb.q[q], ca.q[q], acc, 0, 0, 0);
            } else acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vb[u], va[u], acc, 0, 0, 0, (int)xb[u], 0, (int)xa[u]);
        }
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
    store_one(static_cast<T *>(P.C) + (long long)row * P.ldc + col, v);
}

// ---- launchers -------------------------------------------------------------
// slices of a loop so that there are some 2048 workgroups, where the loop has that many steps
static int slices(long long blocks, int steps)
{
    const long long want = (2048 + blocks - 1) / blocks;
    return (int)(want < 1 ? 1 : want > steps ? steps : want);
}

// What goes past the caches, where rows are whole lines (others share lines, which are better left there).
// An X of 64 to 256 MB, the size of the last cache, when it is quantised: both ways 73 -> 67 us at 16,384 x 5120 bf16; a larger one is not there to begin
// with (75,600 x 5120 both ways 301 us, past the caches 308).
// Values that are written: bf16 from 128 MB on, fp32 from 256 MB on.  Smaller ones are better left there for whoever reads them next, larger ones leave
// them to the codes: written past the caches / through them and quantised again, us, 5120 columns
//   bf16  64 MB 41 / 37   96 MB 55 / 50   128 MB 74 / 73   144 MB 80 / 94   160 MB 85 / 103   240 MB 127 / 143   400 MB 275 / 282
//   fp32  64 MB 49 / 38  128 MB 90 / 70   192 MB 132 / 108  240 MB 171 / 155  320 MB 212 / 223  800 MB 526 / 547
static bool whole_lines(const void *X, int64_t ld, int es) { return (reinterpret_cast<uintptr_t>(X) & 127) == 0 && ld * es % 128 == 0; }

// f(type, STREAM) with both known at compile time
template <typename F> static int with_types(int dtype, bool stream, F f)
{
    if (dtype == SVG2_BF16) stream ? f((bf16_t *)0, std::true_type()) : f((bf16_t *)0, std::false_type());
    else stream ? f((float *)0, std::true_type()) : f((float *)0, std::false_type());
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int fp8_blocks_quant_launch(const void *X, int dtype, int M, int G, int Kg, int64_t sm, int64_t sg, bool square, void *codes, void *scales,
                            void *codes_t, void *scales_t, hipStream_t st)
{
    const int K = G * Kg, es = dtype == SVG2_BF16 ? 2 : 4;
    const bool lines = G == 1 || (sg * es % 128 == 0 && Kg * es % 128 == 0);
    const long long all = (long long)cdiv(M, 128) * cdiv(K, 128);
    const bool shared = !lines || sm * es % 128 != 0 || (reinterpret_cast<uintptr_t>(X) & 127) != 0;
    const BlockQuantArgs A = {X, sm, sg, M, G, Kg, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales),
                              static_cast<uint8_t *>(codes_t), static_cast<uint8_t *>(scales_t), shared ? (int)((all + 7) / 8) : 0};
    const double bytes = (double)M * K * es;
    return with_types(dtype, lines && whole_lines(X, sm, es) && bytes >= 67108864.0 && bytes < 268435456.0, [&](auto *tp, auto stream) {
        using T = std::remove_pointer_t<decltype(tp)>;
        constexpr bool S = decltype(stream)::value;
        if (!codes_t && !square) {
            const int bx = cdiv(M, 16);
            fp8_blocks_rows_kernel<T, S><<<dim3(bx, slices(bx, cdiv(K, 128))), 256, 0, st>>>(A);
            return;
        }
        const long long turns = A.per_xcd ? 8LL * A.per_xcd : all;
        const int tiles = (int)(turns < 1 << 20 ? turns : 1 << 20);
        if (square) {
            if (!codes_t) fp8_blocks_tile_kernel<T, S, true, false, true><<<tiles, 256, 0, st>>>(A);
            else if (!codes) fp8_blocks_tile_kernel<T, S, false, true, true><<<tiles, 256, 0, st>>>(A);
            else fp8_blocks_tile_kernel<T, S, true, true, true><<<tiles, 256, 0, st>>>(A);
        } else if (codes) fp8_blocks_tile_kernel<T, S, true, true, false><<<tiles, 256, 0, st>>>(A);
        else fp8_blocks_tile_kernel<T, S, false, true, false><<<tiles, 256, 0, st>>>(A);
    });
}

int fp8_blocks_values_launch(const void *codes, const void *scales, int M, int K, int dtype, void *X, int64_t ldx, hipStream_t st)
{
    const int es = dtype == SVG2_BF16 ? 2 : 4;
    return with_types(dtype, whole_lines(X, ldx, es) && (double)M * K * es >= 67108864.0 * es, [&](auto *tp, auto stream) {
        using T = std::remove_pointer_t<decltype(tp)>;
        const int bx = cdiv(M, 16);
        fp8_blocks_values_kernel<T, decltype(stream)::value><<<dim3(bx, slices(bx, cdiv(K, 128))), 256, 0, st>>>(
            static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), M, K, static_cast<T *>(X), ldx);
    });
}

using Large = Tile<2, 4, 4, 2>;
using Medium = Tile<2, 2, 2, 2>;
using Small = Tile<2, 2, 1, 1>;

template <typename L> static int prepare_tiles()
{
    SVG2_TRY(set_dynamic_lds(reinterpret_cast<const void *>(&fp8_blocks_product_kernel<L, bf16_t, false>), L::LDS));
    SVG2_TRY(set_dynamic_lds(reinterpret_cast<const void *>(&fp8_blocks_product_kernel<L, float, false>), L::LDS));
    return set_dynamic_lds(reinterpret_cast<const void *>(&fp8_blocks_product_kernel<L, float, true>), L::LDS);
}

int fp8_blocks_matmul_prepare()
{
    SVG2_TRY(prepare_tiles<Large>());
    SVG2_TRY(prepare_tiles<Medium>());
    return prepare_tiles<Small>();
}

static bool few(int M, int N, int K)
{
    return M <= 8 && K <= 8192 && (long long)N * K <= (M <= 4 ? 10LL : 5LL) << 24;
}

// Microseconds that the product takes with these tiles, as measured: `start` a tile, and for each of its `per` stages `full` in a round of as many as fit (a
// CU has 1 large one, 2 medium, 4 small); in a last round that leaves places empty down to `alone`, by how many share a CU in it and by the square of
// its share of all places.  Fitted to 431 sizes from 9 to 30,000 rows, 64 to 16,384 columns and 64 to 80,000 deep, either type of result, up to 27
// combinations of tiles and parts each, and to 84 of 9 to 500 rows whose weights come from memory, for the choice to be right: it takes on average 1.3 % more
// than the best of them, 2.1 % where weights come from memory (numbers of parts: 1 to 6, 8, 11 and 16 of the 16 that it weighs).  Large tiles do most with what they load, small ones leave fewer CUs idle: measured, large / medium /
// small, bf16 results and (fp32)
//   8192 x 8192 x 8192  392 / 469 / 825 us (728 / 853 / 1211)     4096 x 4096 x 4096  55 / 63 / 108 us (102 / 112 / 158)
//   4096 x 5120 x 5120  112 / 104 / 175 us (204 / 167 / 244)      2048 x 2048 x 2048  23 / 13 /  16 us (39 / 22 / 24)
//    512 x 5120 x 5120   50 /  31 /  27 us (86 / 38 / 41)          300 x 5120 x 5120  49 / 29 /  24 us (86 / 36 / 29)
template <typename L> static double tile_time(int M, int N, int per, int split, bool exact)
{
    constexpr int R = L::BM == 256 ? 1 : L::BM == 128 ? 2 : 4;
    const double start = exact ? (R == 1 ? 10.8 : R == 2 ? 3.47 : 1.85) : (R == 1 ? 9.76 : R == 2 ? 3.87 : 3.62);
    const double alone = exact ? (R == 1 ? 2.49 : R == 2 ? 0.863 : 0.450) : (R == 1 ? 1.01 : R == 2 ? 0.508 : 0.321);
    const double full = exact ? (R == 1 ? 2.75 : R == 2 ? 1.64 : 1.20) : (R == 1 ? 1.36 : R == 2 ? 0.822 : 0.658);
    const double by_cu = R == 1 ? 0.0 : exact ? 0.725 : 0.357;
    const long long tiles = (long long)cdiv(M, L::BM) * cdiv(N, L::BN) * split, rounds = tiles / (256 * R), rest = tiles % (256 * R);
    const double share = rest / (256.0 * R), sharing = R == 1 ? 0.0 : (double)((rest + 255) / 256 - 1) / (R > 1 ? R - 1 : 1);
    const double last = alone + (full - alone) * (by_cu * sharing + (1.0 - by_cu) * share * share);
    return (double)rounds * (start + per * full) + (rest ? start + per * last : 0.0);
}

// Which tiles, and in how many parts the contraction: the least time by that model; parts of whole words of scales (four stages), 16 parts at
// most.  Adding them up is a second launch and the parts' way out and back: 2.6 us, and 0.183 us for each MB of the parts.  Measured, one part / as
// chosen, fp32 results (bf16):
//   1536 x 1536 x 16,384  99 / 82 us (70 / 49)     1536 x 1536 x 75,600  466 / 282 us (337 / 169)     512 x 512 x 16,384  55 / 22 us (58 / 19)
// Large tiles go out 256 at a time: the last rows of C, whose tiles would not fill a last round, may be a launch of smaller ones that do
// (75,600 x 5120 x 5120 is 23 rounds and 32 tiles: 1600 us, the 336 last rows by themselves 1560).
struct BlockProductPlan {
    int size, split, per;           // size: 0 small, 1 medium, 2 large
    int rest, rest_size;            // of the rows of C, the last ones that other tiles take
};

static BlockProductPlan product_plan(int M, int N, int K, bool exact)
{
    const int stages = cdiv(K, 128);
    BlockProductPlan best = {0, 1, stages, 0, 0};
    double least = 1e300;
    auto offer = [&](double time, const BlockProductPlan &plan) {
        if (time < least * 0.999) {
            least = time;
            best = plan;
        }
    };
    for (int split = 1; split <= 16 && (split == 1 || stages >= 8 * split); ++split) {
        const int per = split == 1 ? stages : cdiv(cdiv(stages, split), 4) * 4;
        if (split > 1 && (cdiv(stages, per) != split || (double)split * M * N > (1 << 28))) continue;
        const double join = split == 1 ? 0.0 : 2.6 + 0.183 * split * (double)M * N * sizeof(float) * 1e-6;
        offer(join + tile_time<Small>(M, N, per, split, exact), {0, split, per, 0, 0});
        offer(join + tile_time<Medium>(M, N, per, split, exact), {1, split, per, 0, 0});
        offer(join + tile_time<Large>(M, N, per, split, exact), {2, split, per, 0, 0});
    }
    const long long tiles_n = cdiv(N, 256), keep = cdiv(M, 256) * tiles_n / 256 * 256 / tiles_n * 256;      // rows that fill whole rounds
    if (keep >= 256 && keep < M) {
        const int rest = M - (int)keep;
        const double large = tile_time<Large>((int)keep, N, stages, 1, exact) + 2.0;        // and a launch
        offer(large + tile_time<Small>(rest, N, stages, 1, exact), {2, 1, stages, rest, 0});
        offer(large + tile_time<Medium>(rest, N, stages, 1, exact), {2, 1, stages, rest, 1});
    }
    return best;
}

size_t fp8_blocks_matmul_ws_bytes(int M, int N, int K)
{
    if (few(M, N, K)) return 256;
    size_t most = 256;              // of either type of result
    for (bool exact : {false, true}) {
        const BlockProductPlan p = product_plan(M, N, K, exact);
        const size_t need = p.split == 1 ? 256 : (size_t)p.split * M * N * sizeof(float);
        if (need > most) most = need;
    }
    return most;
}

template <typename L, typename T, bool EXACT> static int product_tiles(BlockProductArgs P, hipStream_t st)
{
    P.tiles_n = cdiv(P.N, L::BN);
    const int tiles = cdiv(P.M, L::BM) * P.tiles_n * P.split, resident = 256 * (L::BM == 256 ? 1 : L::BM == 128 ? 2 : 4);
    fp8_blocks_product_kernel<L, T, EXACT><<<tiles < resident ? tiles : resident, 64 * L::WAVES, L::LDS, st>>>(P);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

template <typename T, bool EXACT> static int product_sized(int size, const BlockProductArgs &P, hipStream_t st)
{
    return size == 2 ? product_tiles<Large, T, EXACT>(P, st) : size == 1 ? product_tiles<Medium, T, EXACT>(P, st) : product_tiles<Small, T, EXACT>(P, st);
}

static int product_few(const BlockProductArgs &P, int out_dtype, hipStream_t st)
{
    // 4 wavefronts, 8 or 16: enough of them for the whole card, not more than there are blocks in a row.  Fewer to a workgroup leave others on the CU
    // when some are through: 15,360 x 5120, 16 wavefronts 18.7 us, 8 15.1
    const int blocks = cdiv(P.N, 16);
    int waves = 4;
    while (waves < FEW_WAVES && waves < P.nk && (long long)blocks * waves < 8192) waves *= 2;
    if (out_dtype == SVG2_BF16) fp8_blocks_few_kernel<bf16_t, false><<<blocks, 64 * waves, 0, st>>>(P);
    else fp8_blocks_few_kernel<float, true><<<blocks, 64 * waves, 0, st>>>(P);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int fp8_blocks_matmul_launch(const void *A, const void *SA, const void *B, const void *SB, int M, int N, int K, const float *bias,
                             int out_dtype, void *C, int64_t ldc, void *ws, hipStream_t st)
{
    BlockProductArgs P = {static_cast<const uint8_t *>(A), static_cast<const uint8_t *>(B), static_cast<const uint8_t *>(SA),
                          static_cast<const uint8_t *>(SB), M, N, cdiv(K, 128), M, bias, C, ldc, 0, 1, cdiv(K, 128)};
    if (few(M, N, K)) return product_few(P, out_dtype, st);
    const bool exact = out_dtype == SVG2_F32;
    const BlockProductPlan p = product_plan(M, N, K, exact);
    if (p.split == 1) {
        auto rows = [&](int from, int count, int size) {
            BlockProductArgs part = P;
            part.M = count;
            part.A += (size_t)from * P.nk * 128;
            part.SA += 4 * (size_t)from;
            part.C = static_cast<char *>(C) + (size_t)from * ldc * (exact ? 4 : 2);
            return exact ? product_sized<float, true>(size, part, st) : product_sized<bf16_t, false>(size, part, st);
        };
        SVG2_TRY(rows(0, M - p.rest, p.size));
        return p.rest ? rows(M - p.rest, p.rest, p.rest_size) : SVG2_OK;
    }
    P.split = p.split;
    P.per = p.per;
    BlockProductArgs parts = P;
    parts.bias = nullptr;
    parts.C = ws;
    parts.ldc = N;
    SVG2_TRY(out_dtype == SVG2_BF16 ? (product_sized<float, false>(p.size, parts, st)) : (product_sized<float, true>(p.size, parts, st)));
    const int wide = N % 4 == 0 ? 4 : 1;
    const dim3 grid(cdiv(N, 256 * wide), M < 4096 ? M : 4096);
    const float *from = static_cast<const float *>(ws);
    if (out_dtype == SVG2_BF16) {
        if (wide == 4) fp8_blocks_join_kernel<bf16_t, 4><<<grid, 256, 0, st>>>(from, P);
        else fp8_blocks_join_kernel<bf16_t, 1><<<grid, 256, 0, st>>>(from, P);
    } else {
        if (wide == 4) fp8_blocks_join_kernel<float, 4><<<grid, 256, 0, st>>>(from, P);
        else fp8_blocks_join_kernel<float, 1><<<grid, 256, 0, st>>>(from, P);
    }
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

}  // namespace svg2

// Layer norm of the rows of B groups, with a factor and an offset that all rows share or that each group has for itself (the modulation
// by a timestep), its result as a tensor or as an FP8 operand of the product that follows, and its gradients.
//
//   n  = (x - mean) r,   r = 1 / sqrt(mean((x - mean)^2) + eps),   y = n s + b,   s = w or 1 + w
// backward, with g = dy s:
//   dx = r (g - mean(g) - n mean(g n)),   dw = sum of dy n,   db = sum of dy   over the rows that share them
//
// Every element is read once and written once, some ten operations each: HBM bounds it, where the sums keep out of the way.  A row stays in
// registers between its sums and its result; the mean is taken off before squares are summed.
// 75,600 x 5120 bf16 (1.55 GB in and out) 282 us, 5.5 TB/s, the rate of a large copy; the same as an FP8 operand (1.16 GB) 240 us, 4.8 TB/s:
// instructions, some 15 an element, and one round over the wavefronts a row keep it from 219.  Gradients of 16,384 x 5120 bf16 (0.50 GB) 108 us with
// the sums of the weights', 4.7 TB/s, of 75,600 x 5120 475 us, 4.9 TB/s.
#include <type_traits>

#include "svg2_fp8_blocks.h"

namespace svg2 {

struct NormArgs {
    const void *x, *dy;
    void *y, *dx;                   // y: forward; dx: backward
    long long xs[2], ys[2], ds[2];  // strides of x, of y or dy, of dx: group, row
    const float *w, *b;             // null: 1 (0 where one_plus adds to it), 0
    long long ws, bs;               // their strides from group to group
    int B, N, D;
    float one, eps;                 // one: added to w
    uint8_t *codes, *scales;        // FP8 operand instead of y
    float *dw, *db;                 // gradients, or partial sums: [groups][P][D] each
    int per_group, P;               // backward: whether groups have sums of their own, and parts of a group's rows
};

// Rows whose sums leave fp32's range (an infinity and a NaN among them) are taken again times this: squares of the largest numbers, 16384 of
// them, then stay below 2^126.  Either their squares were too many, which are then above 2^-30; or their sum was, of numbers above 2^113, two of which
// differ by 2^16 then, if any do.  If none do, the row has no variance, as one of zeros.  An eps of up to 1e30 may still count beside the first.
constexpr float SHRINK = 0x1p-72f;
constexpr int WAVES = 16;           // most of a workgroup

__device__ __forceinline__ bool finite(float x) { return mag(x) < 0x7F800000u; }

// x / y by inv, 1 / y rounded: times inv alone, the mean of a constant row would not be that constant
__device__ __forceinline__ float quotient(float x, float y, float inv)
{
    const float q = x * inv;
    return fmaf(fmaf(-q, y, x), inv, q);
}

// sum over 16, 32 or 64 neighbouring lanes, in all of them: no trip through LDS, which takes __shfl_xor some hundred cycles a step.  The same bits in
// every lane, since each step adds what two halves have, either way round: a row's lanes decide by it together whether they go on, to barriers too.
// (Rotated by 4 before 8, half of the lanes would add their neighbours' quads in another order; a product, unless it is rounded first, would be fused
// with the first addition, each lane's own with its neighbour's rounded one.)
template <int LANES> __device__ __forceinline__ float lane_sum(float x)
{
    auto dpp = [](float v, auto control) {
        return __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), decltype(control)::value, 0xF, 0xF, true));
    };
    asm("" : "+v"(x));
    x += dpp(x, std::integral_constant<int, 0xB1>());           // quad_perm [1,0,3,2]
    x += dpp(x, std::integral_constant<int, 0x4E>());           // quad_perm [2,3,0,1]
    x += dpp(x, std::integral_constant<int, 0x128>());          // row_ror:8
    x += dpp(x, std::integral_constant<int, 0x124>());          // row_ror:4
    if constexpr (LANES >= 32) {                                // odd rows of 16 against even ones
        const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    if constexpr (LANES == 64) {                                // the upper half against the lower
        const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    return x;
}

// waits for these loads
template <typename T, int CH> __device__ __forceinline__ void arrived(Raw<T> (&r)[CH])
{
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (unsigned i = 0; i < sizeof(T) / 2; ++i) asm volatile("" : "+v"(r[c].q[i]));
}

// Columns k .. k + 7 of a row of D, in two steps, so that nothing waits where it is loaded: threads at and behind the end of the row load its last eight
// columns, and what is not theirs is moved out when it is used.  (With a branch for each column that is there, the last wavefront had no next row on
// its way: gradients of 16,384 x 5112 bf16 199 us, of 5120 108, now 126 and 104.)  Rows of fewer than eight: column by column.
template <typename T, bool WHOLE, int LANES> __device__ __forceinline__ Raw<T> load_columns(const T *row, int k, int D)
{
    if (WHOLE) return load_raw<T>(row + k);
    if (LANES == 16 && D < 8) return load_raw(row, k, D);
    return load_raw<T>(row + min(k, D - 8));
}

// end: the wavefront reaches the end of the row
template <typename T, bool WHOLE, int LANES> __device__ __forceinline__ void use_columns(const Raw<T> &r, int k, int D, bool end, float *v)
{
    decode<T>(r, v);
    if (WHOLE || !end || (LANES == 16 && D < 8)) return;
    const int s = k - min(k, D - 8);                            // 8 and more: none is there
    if (D & 7)
#pragma unroll
        for (int by = 4; by; by >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = !(s & by) ? v[i] : i + by < 8 ? v[i + by] : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = s < 8 ? v[i] : 0.f;
}

// Gradients of a row that is taken again: the row times SHRINK; or, with true, zeros for a row of one finite number, whose sum need not be a multiple
// of it in fp32.
template <typename TX, int LANES, int CH, bool WHOLE> __device__ __forceinline__ bool take_again(const TX *row, float (&v)[CH][8], int t, int T, int D)
{
    asm volatile("" : "+v"(t), "+s"(D));        // what is formed of them is formed here, not kept in registers through all rows
    const float first = to_f32(row[0]);
    int others = finite(first) && first != 0.f ? 0 : 1;                // columns that differ from the first
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int k = (c * T + t) * 8;
        use_columns<TX, WHOLE, LANES>(load_columns<TX, WHOLE, LANES>(row, k, D), k, D, true, v[c]);
        others += WHOLE ? 8 : min(max(D - k, 0), 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) others -= v[c][i] == first;         // (places behind the end have 0)
    }
    bool same = others == 0;
    if constexpr (LANES) {                                      // of the row's lanes; others may be past their last row
        const unsigned long long other = __ballot(!same) >> (threadIdx.x & 63 & ~(LANES - 1));
        same = (other & (~0ULL >> (64 - LANES))) == 0;
    } else same = __syncthreads_and(same);
    const float by = same ? 0.f : SHRINK;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= by;
    return same;
}

__device__ __forceinline__ void load_weight8(const float *row, int k, int D, float *v)
{
    if (k + 8 <= D) load8<float>(row + k, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < D ? row[k + i] : 0.f;
}

template <typename T> __device__ __forceinline__ void store_row8(T *row, int k, int D, const float *v)
{
    if (k + 8 <= D) store8<T>(row + k, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < D) store_one(row + k + i, v[i]);
}

// One round over the wavefronts of a workgroup for a row's mean and sum of squares.  Each wavefront sums its columns' squares about its own mean;
// of all of them together,
//   mean = sum(n_k mean_k) / D,   squares = sum(squares_k + n_k (mean_k - mean)^2),   sum g (x - mean) = sum(gx_k + (mean_k - mean) g_k)
// which cancels nothing, as sums of x and x^2 would.  Two copies in turn: one is written again only behind a barrier that every thread reaches
// after it has read it.
struct Wave { float mean, squares, g, gx; };

// columns of wavefront k, CH steps of 8 T columns a row
template <int CH> __device__ __forceinline__ float wave_columns(int k, int T, int D)
{
    int n = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) n += min(max(D - (c * T + 64 * k) * 8, 0), 512);
    return (float)n;
}

// mean, squares, g and gx of a row from those of this wavefront.  Every 16 lanes take one wavefront's each.
template <bool GRADIENT> __device__ __forceinline__ void join_waves(Wave &x, Wave *s, int waves, float count, float D, float inv_d)
{
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    // lane % 16, formed here: kept from row to row it went to memory, and the wait for it was one for the next row as well (75,600 x 5120 to FP8 356
    // us, this way 311)
    int k;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0\n\tv_and_b32 %0, 15, %0" : "=v"(k));
    Wave w = {0.f, 0.f, 0.f, 0.f};
    if (k < waves) w = s[k];
    x.mean = quotient(lane_sum<16>(count * w.mean), D, inv_d);
    const float d = k < waves ? w.mean - x.mean : 0.f;
    x.squares = lane_sum<16>(fmaf(count * d, d, w.squares));
    if (GRADIENT) {
        x.g = lane_sum<16>(w.g);
        x.gx = lane_sum<16>(fmaf(d, w.g, w.gx));
    }
}

// sum over the row, in all its threads, of a sum that each has of its columns
template <int LANES> __device__ __forceinline__ float row_sum(float x, Wave (*s)[LANES ? 1 : WAVES], int &copy, int waves)
{
    x = lane_sum<LANES ? LANES : 64>(x);
    if constexpr (!LANES) {
        if ((threadIdx.x & 63) == 0) s[copy][threadIdx.x >> 6].mean = x;
        __syncthreads();
        const int k = threadIdx.x & 15;
        x = lane_sum<16>(k < waves ? s[copy][k].mean : 0.f);
        copy ^= 1;
    }
    return x;
}

// v - mean (0 where there is no column), and the sum of its squares
template <int CH> __device__ __forceinline__ float deviations(float (&v)[CH][8], float mean, int t, int T, int D, bool ragged)
{
    float squares = 0.f;
    auto each = [&](auto by_column) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float m = (c * T + t) * 8 < D ? mean : 0.f;
            asm("" : "+v"(m));      // once for the eight: the compiler would choose between v and v - mean eight times
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] -= !decltype(by_column)::value || (c * T + t) * 8 + i < D ? m : 0.f;
                squares = fmaf(v[c][i], v[c][i], squares);
            }
        }
    };
    if (ragged) each(std::true_type());
    else each(std::false_type());
    return squares;
}

// LANES threads a row, CH steps of 8 columns a thread: 16, 32 or 64 lanes of a block of 256, or (0) a workgroup of up to 512.  A place, the threads
// of a row, goes through neighbouring rows and keeps their factors and offsets in registers: from the caches, they are twice to four times the
// bytes of the rows themselves (75,600 x 5120 bf16 that way 474 us).  The next row is on its way while this one is used.
// WHOLE: rows are as long as the steps of their threads, so that nothing asks where they end.  Wavefronts a SIMD: four at least, five where they fit
// without going to memory (31,299 x 1855 to FP8 with five 45 us, four 42); eight for rows of up to 512 (75,600 x 512 to FP8 with seven 25 us).
template <typename TX, typename TY, bool FP8, int LANES, int CH, bool WHOLE>
__global__ __launch_bounds__(LANES ? 256 : 512, LANES ? (LANES == 64 && CH == 1 && sizeof(TX) == 2 ? 8 : 1) : CH == 2 ? (sizeof(TX) == 2 && (WHOLE || !FP8) ? 5 : 4) : 2) void layer_norm_kernel(const NormArgs A)
{
    __shared__ Wave s_wave[2][LANES ? 1 : WAVES];
    constexpr int PLACES = 256 / (LANES ? LANES : 256);
    const int T = LANES ? LANES : (int)blockDim.x, t = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, D = A.D, nk = (D + 127) / 128;
    const long long rows = (long long)A.B * A.N, places = (long long)gridDim.x * PLACES;
    const long long place = (long long)blockIdx.x * PLACES + (PLACES > 1 ? threadIdx.x / (256 / PLACES) : 0);
    const long long from = rows * place / places, to = rows * (place + 1) / places;
    const bool ragged = !WHOLE && (D & 7);                      // a thread's eight columns are all there or none, but for these lengths
    const float count = (float)D, inv_count = 1.f / count, own = LANES ? count : wave_columns<CH>(threadIdx.x >> 6, T, D);
    const float inv_own = own > 0.f ? 1.f / own : 0.f;
    const float other = LANES ? 0.f : wave_columns<CH>(threadIdx.x & 15, T, D);         // of the wavefront that this lane joins
    const int last = LANES ? LANES : (__builtin_amdgcn_readfirstlane(threadIdx.x) & ~63) + 64;
    float f[CH][8], o[CH][8];
    int group = -1, copy = 0;
    unsigned left_out = 0;                                      // a bit for each row of this place that is taken again
    Raw<TX> next[CH];
    int b = (int)(from / A.N), n = (int)(from - (long long)b * A.N);
    auto load = [&]() {
        const TX *x = static_cast<const TX *>(A.x) + b * A.xs[0] + n * A.xs[1];
#pragma unroll
        for (int c = 0; c < CH; ++c) next[c] = load_columns<TX, WHOLE, LANES>(x, (c * T + t) * 8, D);
    };
    // eight columns of a result
    auto put = [&](long long row, int rb, int rn, int c, const float *v, unsigned byte, const uint2 &codes) {
        const int k = (c * T + t) * 8;
        if constexpr (!FP8) {
            TY *y = static_cast<TY *>(A.y) + rb * A.ys[0] + rn * A.ys[1];
            if (WHOLE) store8<TY>(y + k, v);
            else if (k < D) store_row8(y, k, D, v);
        } else {
            const int kc = k >> 7;
            if (WHOLE || kc < nk) *reinterpret_cast<uint2 *>(A.codes + row * (nk * 128LL) + k) = codes;
            else byte = 0;
            uint8_t *s = A.scales + ((long long)(kc >> 2) * rows + row) * 4;
            if constexpr (LANES == 0 || LANES == 64) {          // a wavefront's step is a word of scales
                const unsigned word = (unsigned)__builtin_amdgcn_readlane((int)byte, 0) | (unsigned)__builtin_amdgcn_readlane((int)byte, 16) << 8 |
                                      (unsigned)__builtin_amdgcn_readlane((int)byte, 32) << 16 | (unsigned)__builtin_amdgcn_readlane((int)byte, 48) << 24;
                if ((t & 63) == 0 && (WHOLE || kc < nk)) *reinterpret_cast<unsigned *>(s) = word;
            } else if ((t & 15) == 0) {
                s[kc & 3] = (uint8_t)byte;
                if (t == 0)                                     // the lanes of a short row do not reach the end of its word
                    for (int z = LANES / 16; z < 4; ++z) s[z] = 0;
            }
        }
    };
    if (from < to) load();
    for (long long row = from; row < to; ++row) {
        const int rb = b, rn = n;
        float v[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) use_columns<TX, WHOLE, LANES>(next[c], (c * T + t) * 8, D, (c * T + last) * 8 > D, v[c]);
        if (++n == A.N) {
            n = 0;
            ++b;
        }
        if (row + 1 < to) load();
        if (rb != group) {
            group = rb;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int k = (c * T + t) * 8;
                if (A.w) load_weight8(A.w + rb * A.ws, k, WHOLE ? k + 8 : D, f[c]);
                if (A.b) load_weight8(A.b + rb * A.bs, k, WHOLE ? k + 8 : D, o[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    f[c][i] = !WHOLE && k + i >= D ? 0.f : A.w ? f[c][i] + A.one : 1.f;
                    o[c][i] = A.b ? o[c][i] : 0.f;
                }
            }
        }
        // v becomes the deviation from the wavefront's own mean, which is `delta` off the row's
        Wave w;
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[c][i];
        const float mean = w.mean = quotient(lane_sum<LANES ? LANES : 64>(sum), own, inv_own);
        w.squares = deviations<CH>(v, mean, t, T, WHOLE ? 1 << 30 : D, ragged);
        w.squares = lane_sum<LANES ? LANES : 64>(w.squares);
        if constexpr (!LANES) {
            join_waves<false>(w, s_wave[copy], T >> 6, other, count, inv_count);
            copy ^= 1;
        }
        const float delta = w.mean - mean;
        bool fine = finite(w.squares);                          // the same for the whole row
        if (LANES == 64) fine = __builtin_amdgcn_readfirstlane(fine);
        if (!fine) left_out |= 1u << (row - from);
        const float r = rsqrtf(fmaf(w.squares, inv_count, A.eps)), shift = -delta * r;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = fmaf(fmaf(v[c][i], r, shift), f[c][i], o[c][i]);
        unsigned bytes[CH] = {};
        uint2 codes[CH] = {};
        if constexpr (FP8) {                                    // 16 lanes a block of 128 columns
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float inv;
                bytes[c] = e4m3_block_scale(max16(largest8(v[c])), inv);
                codes[c] = e4m3_codes8(v[c], inv);
            }
        }
        // The wait for the next row stands in front of this one's stores: behind them it would be a wait for them as well (75,600 x 5120 311 us, here
        // 290; bf16 results, which HBM bounds, 293 and 308)
        if constexpr (FP8) arrived(next);
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (fine) put(row, rb, rn, c, v[c], bytes[c], codes[c]);
    }
    // Rows taken again, behind the loop, where they take no registers from the others (in the loop 600,000 x 64 bf16 38.7 -> 42 us, 75,600 x 512 to FP8
    // 23.3 -> 27).  The mean of numbers that are all the same is off by a few units in the last place, since their sum need not be a multiple of them in
    // fp32; what is left of each of them is the same too, and the sum of that is exact, so that taking its mean off as well leaves zeros.
    for (; left_out; left_out &= left_out - 1) {
        const long long row = from + __builtin_ctz(left_out);
        const int rb = (int)(row / A.N), rn = (int)(row - (long long)rb * A.N);
        const TX *x = static_cast<const TX *>(A.x) + rb * A.xs[0] + rn * A.xs[1];
        float v[CH][8], squares = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            use_columns<TX, WHOLE, LANES>(load_columns<TX, WHOLE, LANES>(x, (c * T + t) * 8, D), (c * T + t) * 8, D, true, v[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] *= SHRINK;
        }
#pragma nounroll
        for (int turn = 0; turn < 2; ++turn) {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += v[c][i];
            squares = deviations<CH>(v, quotient(row_sum<LANES>(sum, s_wave, copy, T >> 6), count, inv_count), t, T, WHOLE ? 1 << 30 : D, ragged);
        }
        squares = row_sum<LANES>(squares, s_wave, copy, T >> 6);
        const float r = rsqrtf(fmaf(squares, inv_count, fmaxf(A.eps * SHRINK * SHRINK, 0x1p-126f)));    // not 0: of a row of one number, r times its zeros is 0
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int k = (c * T + t) * 8;
            float f8[8], o8[8], inv;
            if (A.w) load_weight8(A.w + rb * A.ws, k, WHOLE ? k + 8 : D, f8);
            if (A.b) load_weight8(A.b + rb * A.bs, k, WHOLE ? k + 8 : D, o8);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = !WHOLE && k + i >= D ? 0.f : fmaf(v[c][i] * r, A.w ? f8[i] + A.one : 1.f, A.b ? o8[i] : 0.f);
            const unsigned byte = FP8 ? e4m3_block_scale(max16(largest8(v[c])), inv) : 0;
            put(row, rb, rn, c, v[c], byte, FP8 ? e4m3_codes8(v[c], inv) : uint2());
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// grid: workgroups stride over the shares, P of each group's rows.  LANES threads a row, CH steps of 8 columns a thread: 16 or 32 lanes of a block
// of 64, or (0) the block, a multiple of 64 threads.  A thread keeps its columns' factors and sums; the next row is on its way while this
// one is used.  Wavefronts a SIMD: three at least (31,299 x 1855 fp32 160 us, with two 174), five of one step where a side is bf16 (181,440 x 777 bf16
// 200 us, with four 241).
template <typename TX, typename TY, int LANES, int CH, bool WHOLE>
__global__ __launch_bounds__(LANES ? 64 : 512, CH == 2 ? 3 : !LANES && CH == 1 && sizeof(TX) + sizeof(TY) < 8 ? 5 : 1) void layer_norm_bwd_kernel(const NormArgs A)
{
    constexpr int AT_ONCE = LANES ? 64 / (LANES ? LANES : 64) : 1, SUM = LANES ? LANES : 64;     // rows; lanes of a sum
    __shared__ Wave s_wave[2][WAVES];
    const int T = LANES ? LANES : (int)blockDim.x, t = LANES ? threadIdx.x & (LANES - 1) : threadIdx.x, D = A.D;
    const int groups = A.per_group ? A.B : 1;
    const long long rows = A.per_group ? A.N : (long long)A.B * A.N, shares = (long long)groups * A.P;
    const bool ragged = !WHOLE && (D & 7);
    const float count = (float)D, inv_count = 1.f / count, own = LANES ? count : wave_columns<CH>(t >> 6, T, D), other = LANES ? 0.f : wave_columns<CH>(t & 15, T, D);
    const float inv_own = own > 0.f ? 1.f / own : 0.f;
    const int last = LANES ? LANES : (__builtin_amdgcn_readfirstlane(threadIdx.x) & ~63) + 64;
    int copy = 0;
    for (long long share = blockIdx.x; share < shares; share += gridDim.x) {
        const int group = (int)(share / A.P), part = (int)(share - (long long)group * A.P);
        float acc_w[CH][8], acc_b[CH][8], f[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (A.w) load_weight8(A.w + group * A.ws, (c * T + t) * 8, WHOLE ? (c * T + t) * 8 + 8 : D, f[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc_w[c][i] = acc_b[c][i] = 0.f;
                f[c][i] = A.w ? f[c][i] + A.one : 1.f;
            }
        }
        const long long from = rows * part / A.P + (LANES ? threadIdx.x / SUM : 0), to = rows * (part + 1) / A.P;
        int b = A.per_group ? group : (int)(from / A.N), n = A.per_group ? (int)from : (int)(from - (long long)b * A.N);
        Raw<TX> next_x[CH];
        Raw<TY> next_g[CH];
        auto load = [&]() {
            const TX *x = static_cast<const TX *>(A.x) + b * A.xs[0] + n * A.xs[1];
            const TY *dy = static_cast<const TY *>(A.dy) + b * A.ys[0] + n * A.ys[1];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                next_x[c] = load_columns<TX, WHOLE, LANES>(x, (c * T + t) * 8, D);
                next_g[c] = load_columns<TY, WHOLE, LANES>(dy, (c * T + t) * 8, D);
            }
        };
        if (from < to) load();
        for (long long row = from; row < to; row += AT_ONCE) {
            const int rb = b, rn = n;
            float vx[CH][8], vg[CH][8], gf[CH][8], sg = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const bool end = (c * T + last) * 8 > D;
                use_columns<TX, WHOLE, LANES>(next_x[c], (c * T + t) * 8, D, end, vx[c]);
                use_columns<TY, WHOLE, LANES>(next_g[c], (c * T + t) * 8, D, end, vg[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    gf[c][i] = vg[c][i] * f[c][i];
                    sg += gf[c][i];
                    acc_b[c][i] += vg[c][i];
                }
            }
            sg = lane_sum<SUM>(sg);
            n += AT_ONCE;
            if (!A.per_group)
                while (n >= A.N) {
                    n -= A.N;
                    ++b;
                }
            if (row + AT_ONCE < to) load();
            // vx becomes the deviation from the wavefront's own mean, which is `delta` off the row's
            Wave w;
            float eps = A.eps, scale = 1.f, delta;              // scale: of vx
            for (bool again = false;; again = true) {           // twice where the sums are not finite: the same for the whole row
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += vx[c][i];
                const float mean = w.mean = quotient(lane_sum<SUM>(sum), own, inv_own);
                w.g = sg;
                w.squares = lane_sum<SUM>(deviations<CH>(vx, mean, t, T, WHOLE ? 1 << 30 : D, ragged));
                w.gx = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w.gx = fmaf(gf[c][i], vx[c][i], w.gx);
                w.gx = lane_sum<SUM>(w.gx);
                if (!LANES && T > 64) {
                    join_waves<true>(w, s_wave[copy], T >> 6, other, count, inv_count);
                    copy ^= 1;
                }
                delta = w.mean - mean;
                if (again || finite(w.squares)) break;
                const bool zeros = take_again<TX, LANES, CH, WHOLE>(static_cast<const TX *>(A.x) + rb * A.xs[0] + rn * A.xs[1], vx, t, T, D);
                eps = zeros ? A.eps : A.eps * SHRINK * SHRINK;
                scale = zeros ? 1.f : SHRINK;
            }
            const float r = rsqrtf(fmaf(w.squares, inv_count, eps)), rs = r * scale, shift = -delta * r;
            const float by_n = -(w.gx * r * inv_count) * rs, by_1 = -(w.g * inv_count) * rs;
            TX *dx = static_cast<TX *>(A.dx) + rb * A.ds[0] + rn * A.ds[1];
            arrived(next_x);                                    // in front of the stores, as above
            arrived(next_g);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xn = fmaf(vx[c][i], r, shift);
                    acc_w[c][i] = fmaf(vg[c][i], xn, acc_w[c][i]);
                    v[i] = fmaf(xn, by_n, fmaf(gf[c][i], rs, by_1));
                }
                const int k = (c * T + t) * 8;
                if (WHOLE) store8<TX>(dx + k, v);
                else if (k < D) store_row8(dx, k, D, v);
            }
        }
        if constexpr (LANES) {                                  // the rows that the wavefront had at once
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int other_rows = SUM; other_rows < 64; other_rows <<= 1) {
                        acc_w[c][i] += __shfl_xor(acc_w[c][i], other_rows);
                        acc_b[c][i] += __shfl_xor(acc_b[c][i], other_rows);
                    }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int k = (c * T + t) * 8;
            if (k >= D || (LANES && (int)threadIdx.x >= LANES)) continue;
            if (A.dw) store_row8(A.dw + share * D, k, D, acc_w[c]);
            if (A.db) store_row8(A.db + share * D, k, D, acc_b[c]);
        }
    }
}

// grid (ceil(D / 32), groups by strides, 2), block 1024: dw and db = sum of the P partial sums, 64 bits, always in the same order; 32 threads a column
// take every 32nd.  Bound by its launch and the partial sums (21 MB of 16,384 x 5120: 6 us).
struct NormJoin {
    const float *parts[2];
    float *out[2];
    int D, P, groups;
};

__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const NormJoin J)
{
    __shared__ double s[32][32];
    const int j = threadIdx.x & 31, share = threadIdx.x >> 5, i = blockIdx.x * 32 + j, z = blockIdx.z;
    if (!J.out[z]) return;
    for (int g = blockIdx.y; g < J.groups; g += gridDim.y) {
        double sum = 0.0;
        if (i < J.D) {
            const float *p = J.parts[z] + ((size_t)g * J.P + share) * J.D + i;
#pragma unroll 8
            for (int k = share; k < J.P; k += 32, p += 32 * (size_t)J.D) sum += *p;
        }
        s[share][j] = sum;
        __syncthreads();
        for (int half = 16; half > 0; half >>= 1) {
            if (share < half) s[share][j] += s[share + half][j];
            __syncthreads();
        }
        if (share == 0 && i < J.D) J.out[z][(size_t)g * J.D + i] = (float)s[0][j];
        __syncthreads();
    }
}

// ---- launchers -------------------------------------------------------------
static NormArgs norm_args(const svg2_layer_norm_args *a)
{
    NormArgs A = {};
    A.x = a->x;
    A.y = a->y;
    for (int k = 0; k < 2; ++k) {
        A.xs[k] = a->x_stride[k];
        A.ys[k] = a->y_stride[k];
    }
    A.w = a->weight;
    A.b = a->bias;
    A.ws = a->weight_stride;
    A.bs = a->bias_stride;
    A.B = a->B;
    A.N = a->N;
    A.D = a->D;
    A.one = a->one_plus ? 1.f : 0.f;
    A.eps = a->eps;
    return A;
}

template <typename TX, typename TY, bool FP8> static void norm_forward(const NormArgs &A, hipStream_t st)
{
    const long long rows = (long long)A.B * A.N;
    // Workgroups of `per` places: some rows each, so that factors and offsets are read seldom, but enough of them for the whole card and
    // for places that are through early to be followed by others.  75,600 x 5120 bf16, rows a place: 37 336 us, 18 312, 9 292, 5 288; 16,384 x
    // 5120: 8 71, 4 67, 2 77.  FP8 results leave fewer bytes to hide that reading behind: 75,600 x 5120, 32 rows 253, 16 247, 8 254.
    constexpr int each = FP8 ? 16 : 4;
    auto grid = [&](int per) {
        const long long one = (rows + per - 1) / per, some = (rows + each * per - 1) / (each * per);
        // a launch has fewer than 2^32 threads; a place has 16 rows at most, of 2^26 (the kernel keeps a bit for each)
        return (int)(one < 2048 ? one : some < 2048 ? 2048 : some < 1 << 22 ? some : 1 << 22);
    };
    const int steps = cdiv(A.D, 512);
    // A wavefront a row up to three steps, no barrier: 387M bf16 values in rows of 1536 277 us (FP8 231), by two wavefronts 302 (293); of 1280 309 (271), 362
    // (350).  Whole rows of 5120 280 us (FP8 247), asked for their ends 293 (290); fp32 ones alone are no faster so, 16,384 x 5120 130 against 127.
    constexpr bool whole = FP8 || sizeof(TX) == 2;
    if (A.D <= 128) layer_norm_kernel<TX, TY, FP8, 16, 1, false><<<grid(16), 256, 0, st>>>(A);
    else if (A.D <= 256) layer_norm_kernel<TX, TY, FP8, 32, 1, false><<<grid(8), 256, 0, st>>>(A);
    else if (A.D <= 512) layer_norm_kernel<TX, TY, FP8, 64, 1, false><<<grid(4), 256, 0, st>>>(A);
    else if (A.D <= 1024) layer_norm_kernel<TX, TY, FP8, 64, 2, false><<<grid(4), 256, 0, st>>>(A);
    else if (A.D < 1536) layer_norm_kernel<TX, TY, FP8, 64, 3, false><<<grid(4), 256, 0, st>>>(A);
    else if (A.D == 1536) layer_norm_kernel<TX, TY, FP8, 64, 3, true><<<grid(4), 256, 0, st>>>(A);
    else if (A.D <= 8192 && A.D % 1024 == 0 && whole) layer_norm_kernel<TX, TY, FP8, 0, 2, whole><<<grid(1), steps * 32, 0, st>>>(A);
    else if (A.D <= 8192) layer_norm_kernel<TX, TY, FP8, 0, 2, false><<<grid(1), cdiv(steps, 2) * 64, 0, st>>>(A);
    else layer_norm_kernel<TX, TY, FP8, 0, 4, false><<<grid(1), cdiv(steps, 4) * 64, 0, st>>>(A);
}

int layer_norm_launch(const svg2_layer_norm_args *a, hipStream_t st)
{
    const NormArgs A = norm_args(a);
    const bool x16 = a->dtype == SVG2_BF16, y16 = a->y_dtype == SVG2_BF16;
    if (x16 && y16) norm_forward<bf16_t, bf16_t, false>(A, st);
    else if (x16) norm_forward<bf16_t, float, false>(A, st);
    else if (y16) norm_forward<float, bf16_t, false>(A, st);
    else norm_forward<float, float, false>(A, st);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

int layer_norm_fp8_launch(const svg2_layer_norm_args *a, void *codes, void *scales, hipStream_t st)
{
    NormArgs A = norm_args(a);
    A.codes = static_cast<uint8_t *>(codes);
    A.scales = static_cast<uint8_t *>(scales);
    if (a->dtype == SVG2_BF16) norm_forward<bf16_t, bf16_t, true>(A, st);
    else norm_forward<float, float, true>(A, st);
    SVG2_HIP_CHECK(hipGetLastError());
    return SVG2_OK;
}

// whether the groups' factors or offsets are their own; one group is taken as sharing
static bool per_group(const svg2_layer_norm_args *a)
{
    return a->B > 1 && ((a->weight && a->weight_stride) || (a->bias && a->bias_stride));
}

struct NormBwdPlan {
    bool own;                       // groups have sums of their own
    int lanes, ch, threads, P;      // threads of a row (0: all), their steps of 8 columns, threads; parts of a group's rows
};

// Steps of a thread, one / two, us for 387M bf16 values: rows of 1280 columns 504 / 489, 1536 489 / 482, 2048 495 / 472, 4096 482 / 474; of fewer it depends on
// how many there are: 776 516 / 497, 8192 rows of 776 in fp32 26.9 / 28.5, of 900 30.4 / 32.9, of 1024 29.1 / 25.1.
// Parts: the same number of workgroups for each CU, which else wait for those with one more: 387M values in rows of 4096 in 640 parts 523 us, 768 474,
// 512 473; of 8192 in 320 661, 256 477; of 1280 in 853 705, 1024 603.  As many as a CU holds, by wavefronts: 20 of one step, 12 of two, but 8 where
// no lane is idle (5120 in 512 485, 256 474).  Where there are not half again as many rows, two rows each: more would be more to add up (999 x 777
// in 999 parts 9.3 + 6.4 us, in 500 7.8 + 5.2).
static NormBwdPlan norm_bwd_plan(const svg2_layer_norm_args *a)
{
    NormBwdPlan p;
    p.own = per_group(a);
    p.lanes = a->D <= 128 ? 16 : a->D <= 256 ? 32 : 0;
    p.ch = a->D <= 1024 ? 1 : a->D <= 8192 ? 2 : 4;
    p.threads = cdiv(cdiv(a->D, 512), p.ch) * 64;
    const long long rows = p.own ? a->N : (long long)a->B * a->N, groups = p.own ? a->B : 1;
    const int waves = p.threads / 64, fit = p.ch == 1 ? 20 : p.ch == 4 || a->D % 1024 == 0 ? 8 : 12;
    const long long shares = 256LL * (waves < fit ? fit / waves : 1), at_once = p.lanes ? 64 / p.lanes : 1, turns = (rows + at_once - 1) / at_once;
    const long long parts = shares > groups ? shares / groups : 1;
    p.P = (int)(2 * turns >= 3 * parts ? parts : (turns + 1) / 2);
    return p;
}

size_t layer_norm_bwd_ws_bytes(const svg2_layer_norm_args *a)
{
    const NormBwdPlan p = norm_bwd_plan(a);
    return p.P == 1 || (!a->weight && !a->bias) ? 256 : 2 * align256((size_t)(p.own ? a->B : 1) * p.P * a->D * sizeof(float));
}

int layer_norm_bwd_launch(const svg2_layer_norm_args *a, const void *dY, void *dX, const int64_t *dx_stride, float *dW, float *dB,
                          void *ws, hipStream_t st)
{
    NormArgs A = norm_args(a);
    A.dy = dY;
    A.dx = dX;
    A.ds[0] = dx_stride[0];
    A.ds[1] = dx_stride[1];
    const NormBwdPlan p = norm_bwd_plan(a);
    A.per_group = p.own;
    A.P = p.P;
    const int groups = A.per_group ? A.B : 1;
    if (A.P == 1) {
        A.dw = dW;
        A.db = dB;
    } else {
        A.dw = dW ? static_cast<float *>(ws) : nullptr;
        A.db = dB ? reinterpret_cast<float *>(static_cast<char *>(ws) + align256((size_t)groups * A.P * A.D * sizeof(float))) : nullptr;
    }
    const long long shares = (long long)groups * A.P;
    const int blocks = (int)(shares < 1 << 20 ? shares : 1 << 20);
    auto launch = [&](auto *tx, auto *ty) {
        using TX = std::remove_pointer_t<decltype(tx)>;
        using TY = std::remove_pointer_t<decltype(ty)>;
        if (p.lanes == 16) layer_norm_bwd_kernel<TX, TY, 16, 1, false><<<blocks, 64, 0, st>>>(A);
        else if (p.lanes == 32) layer_norm_bwd_kernel<TX, TY, 32, 1, false><<<blocks, 64, 0, st>>>(A);
        else if (p.ch == 1) layer_norm_bwd_kernel<TX, TY, 0, 1, false><<<blocks, p.threads, 0, st>>>(A);
        else if (p.ch == 2 && A.D % 1024 == 0) layer_norm_bwd_kernel<TX, TY, 0, 2, true><<<blocks, p.threads, 0, st>>>(A);
        else if (p.ch == 2) layer_norm_bwd_kernel<TX, TY, 0, 2, false><<<blocks, p.threads, 0, st>>>(A);
        else layer_norm_bwd_kernel<TX, TY, 0, 4, false><<<blocks, p.threads, 0, st>>>(A);
    };
    const bool x16 = a->dtype == SVG2_BF16, y16 = a->y_dtype == SVG2_BF16;
    if (x16 && y16) launch((bf16_t *)0, (bf16_t *)0);
    else if (x16) launch((bf16_t *)0, (float *)0);
    else if (y16) launch((float *)0, (bf16_t *)0);
    else launch((float *)0, (float *)0);
    SVG2_HIP_CHECK(hipGetLastError());
    if (A.P > 1 && (dW || dB)) {
        const NormJoin J = {{A.dw, A.db}, {dW, dB}, A.D, A.P, groups};
        layer_norm_join_kernel<<<dim3(cdiv(A.D, 32), groups < 1024 ? groups : 1024, 2), 1024, 0, st>>>(J);
        SVG2_HIP_CHECK(hipGetLastError());
    }
    return SVG2_OK;
}

}  // namespace svg2

// Layer norm of the rows of B groups, with a factor and an offset that all rows share or that each group has for itself (the modulation
// by a timestep), its result as a tensor or as an FP8 operand of the product that follows, and its gradients.
//
//   n  = (x - mean) r,   r = 1 / sqrt(mean((x - mean)^2) + eps),   y = n s + b,   s = w or 1 + w
// backward, with g = dy s:
//   dx = r (g - mean(g) - n mean(g n)),   dw = sum of dy n,   db = sum of dy   over the rows that share them
//
// Every element is read once and written once, some ten operations each: HBM bounds it.  A row stays in registers between its sums and its
// result, the mean is taken off before squares are summed.
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
// them, then stay below 2^126, and those of a row that needs it stay above 2^-30, so that eps is nothing beside them.
constexpr float SHRINK = 0x1p-72f;

__device__ __forceinline__ bool finite(float x) { return mag(x) < 0x7F800000u; }

// sum over the LANES threads of a row: 16 or 32 neighbouring lanes, a wavefront, or (LANES > 64) a workgroup, through s
template <int LANES> __device__ __forceinline__ float row_sum(float x, float *s)
{
#pragma unroll
    for (int o = (LANES < 64 ? LANES : 64) >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int k = 0; k < LANES / 64; ++k) x += s[k];
    }
    return x;
}

// eight columns from k on; 0 behind D
template <typename T> __device__ __forceinline__ void load_row8(const T *row, int k, int D, float *v)
{
    if (k + 8 <= D) load8<T>(row + k, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < D ? to_f32(row[k + i]) : 0.f;
}

template <typename T> __device__ __forceinline__ void store_row8(T *row, int k, int D, const float *v)
{
    if (k + 8 <= D) store8<T>(row + k, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < D) store_one(row + k + i, v[i]);
}

// grid: workgroups stride over the rows; block 256, or LANES where a row takes more: LANES threads a row, CH steps of 8 columns a thread
template <typename TX, typename TY, bool FP8, int LANES, int CH>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void layer_norm_kernel(const NormArgs A)
{
    constexpr int BLOCK = LANES < 256 ? 256 : LANES, ROWS = BLOCK / LANES;
    __shared__ float s_sum[4][LANES > 64 ? LANES / 64 : 1];
    const int t = threadIdx.x % LANES, D = A.D, nk = (D + 127) / 128;
    const long long rows = (long long)A.B * A.N;
    const float count = (float)D;               // sums are divided by it: times 1 / D, the mean of a constant row would not be that constant
    for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / LANES; row < rows; row += (long long)gridDim.x * ROWS) {
        const int b = (int)(row / A.N);
        const long long n = row - (long long)b * A.N;
        const TX *x = static_cast<const TX *>(A.x) + b * A.xs[0] + n * A.xs[1];
        float v[CH][8], sum = 0.f, sq = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            load_row8(x, (c * LANES + t) * 8, D, v[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[c][i];
        }
        float eps = A.eps;
        sum = row_sum<LANES>(sum, s_sum[0]);
        if (!finite(sum)) {                                     // the same for the whole row, here and below
            sum = eps = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += v[c][i] *= SHRINK;
            sum = row_sum<LANES>(sum, s_sum[1]);
        }
        const float mean = sum / count;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] = (c * LANES + t) * 8 + i < D ? v[c][i] - mean : 0.f;
                sq = fmaf(v[c][i], v[c][i], sq);
            }
        sq = row_sum<LANES>(sq, s_sum[2]);
        if (!finite(sq)) {
            sq = eps = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[c][i] *= SHRINK;
                    sq = fmaf(v[c][i], v[c][i], sq);
                }
            sq = row_sum<LANES>(sq, s_sum[3]);
        }
        const float r = 1.f / sqrtf(sq / count + eps);
        const float *w = A.w ? A.w + b * A.ws : nullptr, *bias = A.b ? A.b + b * A.bs : nullptr;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int k = (c * LANES + t) * 8;
            float f[8], o[8];
            if (w && k < D) load_row8(w, k, D, f);
            if (bias && k < D) load_row8(bias, k, D, o);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] *= r;
                if (w) v[c][i] *= k + i < D ? f[i] + A.one : 0.f;
                if (bias) v[c][i] += k + i < D ? o[i] : 0.f;
            }
            if constexpr (!FP8) {
                if (k < D) store_row8(static_cast<TY *>(A.y) + b * A.ys[0] + n * A.ys[1], k, D, v[c]);
            } else {                                            // 16 lanes a block of 128 columns
                unsigned top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, mag(v[c][i]));
                float inv;
                const int kc = k >> 7;
                const unsigned byte = e4m3_block_scale(max16(top), inv);
                if (kc < nk) *reinterpret_cast<uint2 *>(A.codes + row * (nk * 128LL) + k) = e4m3_codes8(v[c], inv);
                if ((t & 15) == 0) {
                    uint8_t *s = A.scales + ((long long)(kc >> 2) * rows + row) * 4;
                    if (kc < ((nk + 3) & ~3)) s[kc & 3] = kc < nk ? (uint8_t)byte : 0;
                    if (LANES < 64 && t == 0)                   // the lanes of a short row do not reach the end of its word
                        for (int z = LANES / 16; z < 4; ++z) s[z] = 0;
                }
            }
        }
    }
}

// grid: workgroups stride over the shares, P of each group's rows; block T: a multiple of 64 threads with CH steps of 8 columns each hold
// a row, their columns' factors and sums
template <typename TX, typename TY, int CH> __global__ __launch_bounds__(1024) void layer_norm_bwd_kernel(const NormArgs A)
{
    __shared__ float s_sum[4][2][16];
    const int t = threadIdx.x, T = blockDim.x, waves = T >> 6, wave = t >> 6, D = A.D;
    const int groups = A.per_group ? A.B : 1;
    const long long rows = A.per_group ? A.N : (long long)A.B * A.N, shares = (long long)groups * A.P;
    const float count = (float)D;
    // sums over the workgroup of two values at once; `copy`: another one each time, until a barrier later
    auto sums = [&](float &a, float &b, int copy) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            a += __shfl_xor(a, o);
            b += __shfl_xor(b, o);
        }
        if ((t & 63) == 0) {
            s_sum[copy][0][wave] = a;
            s_sum[copy][1][wave] = b;
        }
        __syncthreads();
        a = b = 0.f;
        for (int k = 0; k < waves; ++k) {
            a += s_sum[copy][0][k];
            b += s_sum[copy][1][k];
        }
    };
    for (long long share = blockIdx.x; share < shares; share += gridDim.x) {
        const int group = (int)(share / A.P), part = (int)(share - (long long)group * A.P);
        float acc_w[CH][8], acc_b[CH][8], f[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (A.w) load_row8(A.w + group * A.ws, (c * T + t) * 8, D, f[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc_w[c][i] = acc_b[c][i] = 0.f;
                f[c][i] = A.w ? f[c][i] + A.one : 1.f;
            }
        }
        const long long from = rows * part / A.P, to = rows * (part + 1) / A.P;
        for (long long row = from; row < to; ++row) {
            const long long b = A.per_group ? group : row / A.N, n = A.per_group ? row : row - b * A.N;
            const TX *x = static_cast<const TX *>(A.x) + b * A.xs[0] + n * A.xs[1];
            const TY *dy = static_cast<const TY *>(A.dy) + b * A.ys[0] + n * A.ys[1];
            float vx[CH][8], vg[CH][8], sx = 0.f, sg = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int k = (c * T + t) * 8;
                load_row8(x, k, D, vx[c]);
                load_row8(dy, k, D, vg[c]);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sx += vx[c][i];
                    acc_b[c][i] += vg[c][i];
                    sg = fmaf(vg[c][i], f[c][i], sg);
                }
            sums(sx, sg, 0);
            float eps = A.eps, scale = 1.f;                     // of vx
            if (!finite(sx)) {
                float none = sx = eps = 0.f;
                scale = SHRINK;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sx += vx[c][i] *= SHRINK;
                sums(sx, none, 1);
            }
            const float mean = sx / count, mean_g = sg / count;
            float sxx = 0.f, sgx = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    vx[c][i] = (c * T + t) * 8 + i < D ? vx[c][i] - mean : 0.f;
                    sxx = fmaf(vx[c][i], vx[c][i], sxx);
                    sgx = fmaf(vg[c][i] * f[c][i], vx[c][i], sgx);
                }
            sums(sxx, sgx, 2);
            if (!finite(sxx)) {
                sxx = sgx = eps = 0.f;
                scale *= SHRINK;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        vx[c][i] *= SHRINK;
                        sxx = fmaf(vx[c][i], vx[c][i], sxx);
                        sgx = fmaf(vg[c][i] * f[c][i], vx[c][i], sgx);
                    }
                sums(sxx, sgx, 3);
            }
            const float r = 1.f / sqrtf(sxx / count + eps), mean_gn = sgx * r / count;
            TX *dx = static_cast<TX *>(A.dx) + b * A.ds[0] + n * A.ds[1];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xn = vx[c][i] * r;
                    acc_w[c][i] = fmaf(vg[c][i], xn, acc_w[c][i]);
                    v[i] = r * scale * (vg[c][i] * f[c][i] - mean_g - xn * mean_gn);
                }
                const int k = (c * T + t) * 8;
                if (k < D) store_row8(dx, k, D, v);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int k = (c * T + t) * 8;
            if (k >= D) continue;
            if (A.dw) store_row8(A.dw + share * D, k, D, acc_w[c]);
            if (A.db) store_row8(A.db + share * D, k, D, acc_b[c]);
        }
    }
}

// grid (ceil(D / 64), groups by strides, 2), block 1024: dw and db = sum of the P partial sums, 64 bits; 16 wavefronts take every 16th
struct NormJoin {
    const float *parts[2];
    float *out[2];
    int D, P, groups;
};

__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const NormJoin J)
{
    __shared__ double s[16][64];
    const int j = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + j, z = blockIdx.z;
    if (!J.out[z]) return;
    for (int g = blockIdx.y; g < J.groups; g += gridDim.y) {
        double sum = 0.0;
        if (i < J.D) {
            const float *p = J.parts[z] + ((size_t)g * J.P + wave) * J.D + i;
#pragma unroll 8
            for (int k = wave; k < J.P; k += 16, p += 16 * (size_t)J.D) sum += *p;
        }
        s[wave][j] = sum;
        __syncthreads();
        if (wave == 0 && i < J.D) {
            for (int k = 1; k < 16; ++k) sum += s[k][j];
            J.out[z][(size_t)g * J.D + i] = (float)sum;
        }
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
    auto grid = [&](int per) { return (int)((rows + per - 1) / per < (1 << 20) ? (rows + per - 1) / per : 1 << 20); };
    if (A.D <= 128) layer_norm_kernel<TX, TY, FP8, 16, 1><<<grid(16), 256, 0, st>>>(A);
    else if (A.D <= 256) layer_norm_kernel<TX, TY, FP8, 32, 1><<<grid(8), 256, 0, st>>>(A);
    else if (A.D <= 512) layer_norm_kernel<TX, TY, FP8, 64, 1><<<grid(4), 256, 0, st>>>(A);
    else if (A.D <= 1024) layer_norm_kernel<TX, TY, FP8, 64, 2><<<grid(4), 256, 0, st>>>(A);
    else if (A.D <= 2048) layer_norm_kernel<TX, TY, FP8, 256, 1><<<grid(1), 256, 0, st>>>(A);
    else if (A.D <= 4096) layer_norm_kernel<TX, TY, FP8, 256, 2><<<grid(1), 256, 0, st>>>(A);
    else if (A.D <= 6144) layer_norm_kernel<TX, TY, FP8, 256, 3><<<grid(1), 256, 0, st>>>(A);
    else if (A.D <= 8192) layer_norm_kernel<TX, TY, FP8, 1024, 1><<<grid(1), 1024, 0, st>>>(A);
    else layer_norm_kernel<TX, TY, FP8, 1024, 2><<<grid(1), 1024, 0, st>>>(A);
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

static int norm_parts(const svg2_layer_norm_args *a)
{
    const bool own = per_group(a);
    const long long rows = own ? a->N : (long long)a->B * a->N;
    long long parts = own ? (1024 + a->B - 1) / a->B : 1024;
    if (parts > (rows + 3) / 4) parts = (rows + 3) / 4;
    return (int)parts;
}

size_t layer_norm_bwd_ws_bytes(const svg2_layer_norm_args *a)
{
    const int P = norm_parts(a);
    return P == 1 ? 256 : 2 * align256((size_t)(per_group(a) ? a->B : 1) * P * a->D * sizeof(float));
}

int layer_norm_bwd_launch(const svg2_layer_norm_args *a, const void *dY, void *dX, const int64_t *dx_stride, float *dW, float *dB,
                          void *ws, hipStream_t st)
{
    NormArgs A = norm_args(a);
    A.dy = dY;
    A.dx = dX;
    A.ds[0] = dx_stride[0];
    A.ds[1] = dx_stride[1];
    A.per_group = per_group(a);
    A.P = norm_parts(a);
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
    const int steps = cdiv(A.D, 512), threads = A.D <= 512 ? 64 : cdiv(steps, 2) * 64;
    auto launch = [&](auto *tx, auto *ty) {
        using TX = std::remove_pointer_t<decltype(tx)>;
        using TY = std::remove_pointer_t<decltype(ty)>;
        if (A.D <= 512) layer_norm_bwd_kernel<TX, TY, 1><<<blocks, threads, 0, st>>>(A);
        else layer_norm_bwd_kernel<TX, TY, 2><<<blocks, threads, 0, st>>>(A);
    };
    const bool x16 = a->dtype == SVG2_BF16, y16 = a->y_dtype == SVG2_BF16;
    if (x16 && y16) launch((bf16_t *)0, (bf16_t *)0);
    else if (x16) launch((bf16_t *)0, (float *)0);
    else if (y16) launch((float *)0, (bf16_t *)0);
    else launch((float *)0, (float *)0);
    SVG2_HIP_CHECK(hipGetLastError());
    if (A.P > 1 && (dW || dB)) {
        const NormJoin J = {{A.dw, A.db}, {dW, dB}, A.D, A.P, groups};
        layer_norm_join_kernel<<<dim3(cdiv(A.D, 64), groups < 1024 ? groups : 1024, 2), 1024, 0, st>>>(J);
        SVG2_HIP_CHECK(hipGetLastError());
    }
    return SVG2_OK;
}

}  // namespace svg2

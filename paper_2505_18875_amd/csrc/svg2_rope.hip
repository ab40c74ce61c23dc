// From a projection's rows to the layer's operands: RMS norm of Q and K, rotary positions over several axes, token order
// -> head order, and the gradients of that.
//
//   n      = x * rsqrt(mean(x^2) + eps) * w         mean over the head, or over all heads of the token
//   y[i,j] = (n[i] cos a - n[j] sin a,  n[i] sin a + n[j] cos a)     pair p = (i,j), a = pos[axis(p)] * freq[p]
// backward, with g = dy turned by -a:
//   dw = sum over tokens (and heads) of g n / w,   dx = r (g w - x r mean(g w x r)),   r = rsqrt(mean(x^2) + eps)
//
// Every element is read once and written once, some ten operations each: HBM bounds it, so the kernels are built around the
// loads.  One wavefront (fewer lanes where a token is short, a workgroup where it is long) per token and tensor; a lane holds
// four pairs (8 elements), 8 or 16 lanes a head, 8 or 4 heads a step, and up to CH steps are loaded before the first is used.  A
// token of 40 heads of 128 thus stays in registers between the sum of squares over all its heads and the result, and no lane
// needs an element of another's.  The angle of a lane's pairs is the same for every head, so four cosines and sines per lane and
// token serve all of them: cheap enough to compute in place, in 64 bits up to the quarter turn (positions of 10^6 times a
// frequency of 1 leave no fraction in 32), instead of reading a table.
// Q, K and V of 75,600 tokens of 40 heads of 128 in bf16 (4.6 GB in and out): 859 to 887 us, 5.2 to 5.4 TB/s, the rate of a large copy.
#include <type_traits>

#include "svg2_common.h"

namespace svg2 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct RopeArgs {
    const void *src[3];             // forward: x; backward: x (null where the tensor has no norm)
    const void *grad[3];            // backward: dy
    void *dst[3];                   // forward: y; backward: dx
    const float *weight[3];         // fp32 [d] or [H,d], null: no norm
    long long ss[3], gs[3], ds[3];  // strides of src, grad, dst: batch, token, head
    const int32_t *pos;
    long long pos_b;
    const double *freq;
    int n_axes, end[4];             // pairs of axis k: end[k-1] .. end[k]
    int rotate;                     // bit t: tensor t is rotated
    int B, N, H, token_scope;
    float eps, sense;               // sense: 1, or -1 to turn back
    float *rinv;                    // backward, long token rows: 1 / rms of every token, [3][B N]
    float *partial;                 // backward: partial sums of dw, [3][P][cols]
    float *dw[3];
    int P, cols;
};

// ---- four pairs of a lane --------------------------------------------------
template <typename T> struct Raw { uint4 q[sizeof(T) / 2]; };

template <typename T, int D, bool ADJ> __device__ __forceinline__ Raw<T> load_pairs(const T *head, int c)
{
    Raw<T> r;
    if constexpr (ADJ) {
#pragma unroll
        for (unsigned k = 0; k < sizeof(T) / 2; ++k) r.q[k] = reinterpret_cast<const uint4 *>(head + 8 * c)[k];
    } else if constexpr (sizeof(T) == 4) {
        r.q[0] = *reinterpret_cast<const uint4 *>(head + 4 * c);
        r.q[1] = *reinterpret_cast<const uint4 *>(head + D / 2 + 4 * c);
    } else {
        const uint2 a = *reinterpret_cast<const uint2 *>(head + 4 * c), b = *reinterpret_cast<const uint2 *>(head + D / 2 + 4 * c);
        r.q[0] = make_uint4(a.x, a.y, b.x, b.y);
    }
    return r;
}

template <typename T, int D, bool ADJ> __device__ __forceinline__ void store_pairs(T *head, int c, const Raw<T> &r)
{
    if constexpr (ADJ) {
#pragma unroll
        for (unsigned k = 0; k < sizeof(T) / 2; ++k) reinterpret_cast<uint4 *>(head + 8 * c)[k] = r.q[k];
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4 *>(head + 4 * c) = r.q[0];
        *reinterpret_cast<uint4 *>(head + D / 2 + 4 * c) = r.q[1];
    } else {
        *reinterpret_cast<uint2 *>(head + 4 * c) = make_uint2(r.q[0].x, r.q[0].y);
        *reinterpret_cast<uint2 *>(head + D / 2 + 4 * c) = make_uint2(r.q[0].z, r.q[0].w);
    }
}

// the eight elements in the order they are stored in; element e of pair k is v[at(k, e)]
template <bool ADJ> __device__ constexpr int at(int k, int e) { return ADJ ? 2 * k + e : 4 * e + k; }

template <typename T> __device__ __forceinline__ void decode(const Raw<T> &r, float *v)
{
#pragma unroll
    for (unsigned k = 0; k < sizeof(T) / 2; ++k) {
        const unsigned w[4] = {r.q[k].x, r.q[k].y, r.q[k].z, r.q[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                v[4 * k + i] = __uint_as_float(w[i]);
            } else {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    }
}

// the one rounding of a bf16 result (to nearest even; NaN stays NaN)
template <typename T> __device__ __forceinline__ Raw<T> encode(const float *v)
{
    Raw<T> r;
    if constexpr (sizeof(T) == 4) {
        r.q[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        r.q[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 p = {v[2 * i], v[2 * i + 1]};
            w[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
        }
        r.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return r;
}

template <int D, bool ADJ> __device__ __forceinline__ void load_weight(const float *w, int c, float *v)
{
    const float4 a = *reinterpret_cast<const float4 *>(w + (ADJ ? 8 * c : 4 * c));
    const float4 b = *reinterpret_cast<const float4 *>(w + (ADJ ? 8 * c + 4 : D / 2 + 4 * c));
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// cosine and sine of the angle of pair p; of the four of a lane.  The quarter turns are taken off in 64 bits (two-part pi / 2: the error is
// that of the product pos * freq itself), what remains is at most pi / 4 and goes through the Taylor polynomials, whose next
// terms there are 2e-9 (sine, x^11 / 11!) and 1e-10 (cosine, x^12 / 12!).
__device__ __forceinline__ void angle(const RopeArgs &A, const int32_t *pos, int p, float &cs, float &sn)
{
    int axis = 0;
#pragma unroll
    for (int x = 0; x < 3; ++x) axis += (x + 1 < A.n_axes && p >= A.end[x]) ? 1 : 0;
    const double t = (double)pos[axis] * A.freq[p];
    const double q = rint(t * 0.63661977236758134);
    const float r = (float)fma(-q, 6.123233995736766e-17, fma(-q, 1.5707963267948966, t));
    const int quadrant = (int)(q - 4.0 * floor(q * 0.25));
    const float z = r * r;
    const float s = r + r * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
    const float co = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 - z * (1.f / 3628800)))));
    const float u = (quadrant & 1) ? s : co, v = (quadrant & 1) ? co : s;
    cs = (quadrant == 1 || quadrant == 2) ? -u : u;
    sn = quadrant >= 2 ? -v : v;
}

__device__ __forceinline__ const int32_t *position(const RopeArgs &A, int b, int n)
{
    return A.pos + (long long)b * A.pos_b + (long long)n * A.n_axes;
}

__device__ __forceinline__ void angles(const RopeArgs &A, int b, int n, int c, float *cs, float *sn)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) angle(A, position(A, b, n), 4 * c + k, cs[k], sn[k]);
}

// A sine of 0 is that of an angle of 0, or below 2^-150 (no other double comes that near to a multiple of pi / 2): such a pair is left as it
// is, since 0 times an infinity would make its partner NaN, and 0 times a negative number, taken off, a negative zero positive.
template <bool ADJ> __device__ __forceinline__ void turn(float *v, const float *cs, const float *sn, float sense)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a = v[at<ADJ>(k, 0)], b = v[at<ADJ>(k, 1)], s = sense * sn[k];
        v[at<ADJ>(k, 0)] = s == 0.f ? a : a * cs[k] - b * s;
        v[at<ADJ>(k, 1)] = s == 0.f ? b : a * s + b * cs[k];
    }
}

// sum over groups of `width` lanes (8, 16: a head; 64: the wavefront)
__device__ __forceinline__ float group_sum(float x, int width)
{
    for (int o = width >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// ---- forward ---------------------------------------------------------------
// grid (ceil(B N / (256 / G)), tensors, 1), block 256: G lanes a token.  64, or where a token has fewer than 512 values the 8, 16 or 32
// that hold them: one head of 64 a wavefront, 4096 tokens, took 11 us, eight of them take 5.  More than 2^23 workgroups go on in the
// third dimension (see token_grid).
template <typename T, int D, bool ADJ, int G, int CH> __global__ __launch_bounds__(256) void rope_kernel(const RopeArgs A)
{
    constexpr int LPH = D / 8, HPS = G / LPH;
    const int lane = threadIdx.x % G, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = (blockIdx.z * gridDim.x + blockIdx.x) * (256 / G) + (G == 64 ? wave : (int)threadIdx.x / G), t = blockIdx.y;
    if (token >= A.B * A.N) return;             // all lanes of a token together: the sums below stay inside them
    const int b = token / A.N, n = token - b * A.N;
    const int hl = lane / LPH, c = lane % LPH;
    const T *src = static_cast<const T *>(A.src[t]) + b * A.ss[0] + n * A.ss[1];
    T *dst = static_cast<T *>(A.dst[t]) + b * A.ds[0] + n * A.ds[1];
    const float *weight = A.weight[t];
    const bool rotate = (A.rotate >> t) & 1, whole = weight && A.token_scope;
    const int steps = (A.H + HPS - 1) / HPS;

    Raw<T> raw[CH];
    auto load = [&](int s0) {
#pragma unroll
        for (int s = 0; s < CH; ++s) {
            const int h = (s0 + s) * HPS + hl;
            if (h < A.H) raw[s] = load_pairs<T, D, ADJ>(src + h * A.ss[2], c);
        }
    };
    float cs[4], sn[4], w[8], rinv = 1.f;
    if (whole) {
        float sum = 0.f;
        for (int s0 = 0; s0 < steps; s0 += CH) {
            load(s0);
            if (s0 == 0 && rotate) angles(A, b, n, c, cs, sn);      // while they come
#pragma unroll
            for (int s = 0; s < CH; ++s) {
                float v[8];
                decode(raw[s], v);
                if ((s0 + s) * HPS + hl < A.H)
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum = fmaf(v[k], v[k], sum);
            }
        }
        rinv = 1.f / sqrtf(group_sum(sum, G) / ((float)A.H * D) + A.eps);
    } else {
        load(0);
        if (weight) load_weight<D, ADJ>(weight, c, w);
        if (rotate) angles(A, b, n, c, cs, sn);
    }
    for (int s0 = 0; s0 < steps; s0 += CH) {
        if (s0 > 0 || (whole && steps > CH)) load(s0);
#pragma unroll
        for (int s = 0; s < CH; ++s) {
            const int h = (s0 + s) * HPS + hl;
            if ((s0 + s) * HPS >= A.H) continue;
            if (weight || rotate) {
                float v[8];
                decode(raw[s], v);
                if (weight) {
                    if (whole) {
                        if (h < A.H) load_weight<D, ADJ>(weight + h * D, c, w);
                    } else {
                        float sum = 0.f;
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum = fmaf(v[k], v[k], sum);
                        rinv = 1.f / sqrtf(group_sum(sum, LPH) * (1.f / D) + A.eps);
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = v[k] * rinv * w[k];
                }
                if (rotate) turn<ADJ>(v, cs, sn, A.sense);
                raw[s] = encode<T>(v);
            }
            if (h < A.H) store_pairs<T, D, ADJ>(dst + h * A.ds[2], c, raw[s]);
        }
    }
}

// Long tokens, not too many: grid (B N, tensors), block 256.  A workgroup takes a token, S steps of 2048 values, so that everything
// it reads is asked for at once; its angles, one a thread, and the sum of squares go round through LDS.
// Measured, us for Q, K and V of 40 heads of 128, this kernel / rope_kernel: 1 token 3.8 / 7.5, 256: 5.2 / 8.9, 1024: 11.5 / 15.2,
// 4096: 38 / 43, 16,384: 205 / 202, 75,600: 938 / 862; 32 heads, 8192 tokens: 77 / 84.
template <typename T, int D, bool ADJ, int S> __global__ __launch_bounds__(256) void rope_row_kernel(const RopeArgs A)
{
    constexpr int LPH = D / 8, HPS = 256 / LPH;
    __shared__ __attribute__((aligned(16))) float s_cs[D / 2], s_sn[D / 2];
    __shared__ float s_sum[4];
    const int tid = threadIdx.x, token = blockIdx.x, t = blockIdx.y, hl = tid / LPH, c = tid % LPH;
    const int b = token / A.N, n = token - b * A.N;
    const T *src = static_cast<const T *>(A.src[t]) + b * A.ss[0] + n * A.ss[1];
    T *dst = static_cast<T *>(A.dst[t]) + b * A.ds[0] + n * A.ds[1];
    const float *weight = A.weight[t];
    const bool rotate = (A.rotate >> t) & 1;
    Raw<T> raw[S];
    float w[S][8], sum = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int h = s * HPS + hl;
        if (h >= A.H) continue;
        raw[s] = load_pairs<T, D, ADJ>(src + h * A.ss[2], c);
        if (weight) load_weight<D, ADJ>(weight + (A.token_scope ? h * D : 0), c, w[s]);
    }
    if (rotate && tid < D / 2) angle(A, position(A, b, n), tid, s_cs[tid], s_sn[tid]);
    if (weight && A.token_scope) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float v[8];
            decode(raw[s], v);
            if (s * HPS + hl < A.H)
#pragma unroll
                for (int k = 0; k < 8; ++k) sum = fmaf(v[k], v[k], sum);
        }
        sum = group_sum(sum, 64);
        if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
    }
    __syncthreads();
    float cs[4], sn[4], rinv = 1.f;
    if (weight && A.token_scope) rinv = 1.f / sqrtf(((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3])) / ((float)A.H * D) + A.eps);
    if (rotate) {
        const float4 u = *reinterpret_cast<const float4 *>(&s_cs[4 * c]), v = *reinterpret_cast<const float4 *>(&s_sn[4 * c]);
        cs[0] = u.x; cs[1] = u.y; cs[2] = u.z; cs[3] = u.w;
        sn[0] = v.x; sn[1] = v.y; sn[2] = v.z; sn[3] = v.w;
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int h = s * HPS + hl;
        if (h >= A.H) continue;                 // whole heads: the sum below stays inside one
        if (weight || rotate) {
            float v[8];
            decode(raw[s], v);
            if (weight) {
                if (!A.token_scope) {
                    float x2 = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) x2 = fmaf(v[k], v[k], x2);
                    rinv = 1.f / sqrtf(group_sum(x2, LPH) * (1.f / D) + A.eps);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = v[k] * rinv * w[s][k];
            }
            if (rotate) turn<ADJ>(v, cs, sn, A.sense);
            raw[s] = encode<T>(v);
        }
        store_pairs<T, D, ADJ>(dst + h * A.ds[2], c, raw[s]);
    }
}

// ---- backward --------------------------------------------------------------
// How the weights' gradient is summed: per lane over the tokens that pass through it, over the block's wavefronts in LDS where
// they hold the same columns, over the blocks by rope_dw_kernel, each in a fixed order, so that it is the same from run to run.  The first
// two in fp32, where a lane's additions in a row grow with the tokens (821 of them for 420,000 tokens of 40 heads of 128 under a norm over the
// token, each off by 2^-24 of the sum at most); over the blocks in 64 bits.
enum { DW_NONE, DW_STEP, DW_ROW, DW_LONG };
//   DW_NONE    no norm: the forward's kernels, turning back
//   DW_STEP    [d] weights, or [H,d] of a token that is one step of a wavefront: 8 sums per lane (rope_bwd_kernel)
//   DW_ROW     longer tokens, up to 8192 [H,d] weights: a wavefront (up to 2048) or a workgroup holds a token, its weights and its sums
//              (rope_bwd_row_kernel).  One wavefront does not hold a token of 5120 values and their sums: 1032 us for Q, K and V of
//              16,384 tokens, most of it spilled registers; the workgroup 294
//   DW_LONG    tokens longer than that: read twice here (sums, then results); 1 / rms is left for rope_dw_long_kernel
constexpr int ROW_STEPS = 4;        // most steps of 8 values a thread that are held

template <int D, bool ADJ> __device__ __forceinline__ int column(int c, int k)     // where value k of lane c is in its head
{
    return ADJ ? 8 * c + k : (k < 4 ? 4 * c + k : D / 2 + 4 * c + k - 4);
}

// adds the block's four wavefronts' sums in order into s[cols]
template <int D, bool ADJ> __device__ __forceinline__ void add_to(float *s, int c, const float *v, bool first)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int i = column<D, ADJ>(c, k);
        s[i] = first ? v[k] : s[i] + v[k];
    }
}

// sums of a lane's share: x^2 and g w x
__device__ __forceinline__ void add_sums(const float *vx, const float *vg, const float *w, float &xx, float &gx)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        xx = fmaf(vx[k], vx[k], xx);
        gx = fmaf(vg[k] * w[k], vx[k], gx);
    }
}

// vg: g on entry, dx on return; acc += g xn (add: this lane has a head)
__device__ __forceinline__ void norm_gradient(const float *vx, float *vg, const float *w, float rinv, float mean, float *acc, bool add)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float xn = vx[k] * rinv;
        if (add) acc[k] += vg[k] * xn;
        vg[k] = rinv * (vg[k] * w[k] - xn * mean);
    }
}

// grid (blocks, tensors), block 256: G lanes a token (64, or the 8, 16 or 32 that hold it), wavefronts stride over the tokens
template <typename T, int D, bool ADJ, int DW, int G> __global__ __launch_bounds__(256, 2) void rope_bwd_kernel(const RopeArgs A)
{
    constexpr int LPH = D / 8, HPS = G / LPH, CH = G < 64 ? 1 : DW == DW_LONG ? 2 : 4;
    __shared__ float s_dw[512];                 // DW_STEP
    const int lane = threadIdx.x % G, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = blockIdx.y;
    const int hl = lane / LPH, c = lane % LPH, steps = (A.H + HPS - 1) / HPS, tokens = A.B * A.N;
    const float *weight = A.weight[t];
    const bool rotate = (A.rotate >> t) & 1, whole = A.token_scope;         // DW_STEP, whole: one step

    float acc[8], w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = 0.f;
    if (DW == DW_STEP && weight && (!whole || hl < A.H)) load_weight<D, ADJ>(weight + (whole ? hl * D : 0), c, w);

    for (int token = blockIdx.x * (256 / G) + (G == 64 ? wave : (int)threadIdx.x / G); token < tokens; token += gridDim.x * (256 / G)) {
        const int b = token / A.N, n = token - b * A.N;
        const T *x = static_cast<const T *>(A.src[t]) + b * A.ss[0] + n * A.ss[1];
        const T *g = static_cast<const T *>(A.grad[t]) + b * A.gs[0] + n * A.gs[1];
        T *dx = static_cast<T *>(A.dst[t]) + b * A.ds[0] + n * A.ds[1];
        Raw<T> rg[CH], rx[CH];
        auto load = [&](int s0) {
#pragma unroll
            for (int s = 0; s < CH; ++s) {
                const int h = (s0 + s) * HPS + hl;
                if (h >= A.H) continue;
                rg[s] = load_pairs<T, D, ADJ>(g + h * A.gs[2], c);
                if (weight) rx[s] = load_pairs<T, D, ADJ>(x + h * A.ss[2], c);
            }
        };
        float cs[4], sn[4], rinv = 1.f, mean = 0.f;
        if (DW == DW_LONG && weight) {
            float xx = 0.f, gx = 0.f;
            for (int s0 = 0; s0 < steps; s0 += CH) {
                load(s0);
                if (s0 == 0 && rotate) angles(A, b, n, c, cs, sn);
#pragma unroll
                for (int s = 0; s < CH; ++s) {
                    const int h = (s0 + s) * HPS + hl;
                    if (h >= A.H) continue;
                    float vx[8], vg[8];
                    decode(rx[s], vx);
                    decode(rg[s], vg);
                    if (rotate) turn<ADJ>(vg, cs, sn, A.sense);
                    load_weight<D, ADJ>(weight + h * D, c, w);
                    add_sums(vx, vg, w, xx, gx);
                }
            }
            const float count = (float)A.H * D;
            rinv = 1.f / sqrtf(group_sum(xx, 64) / count + A.eps);
            mean = group_sum(gx, 64) * rinv / count;
            if (lane == 0) A.rinv[(size_t)t * tokens + token] = rinv;
        } else if (rotate) {
            angles(A, b, n, c, cs, sn);
        }
        for (int s0 = 0; s0 < steps; s0 += CH) {
            load(s0);
#pragma unroll
            for (int s = 0; s < CH; ++s) {
                const int h = (s0 + s) * HPS + hl;
                if ((s0 + s) * HPS >= A.H) continue;
                if (weight || rotate) {
                    float vg[8];
                    decode(rg[s], vg);
                    if (rotate) turn<ADJ>(vg, cs, sn, A.sense);
                    if (weight) {
                        float vx[8];
                        decode(rx[s], vx);
                        if (DW == DW_STEP) {
                            float xx = 0.f, gx = 0.f;
                            if (h < A.H) add_sums(vx, vg, w, xx, gx);
                            const float count = whole ? (float)A.H * D : (float)D;
                            if (whole) {
                                xx = group_sum(xx, G);
                                gx = group_sum(gx, G);
                            } else {
                                xx = group_sum(xx, LPH);
                                gx = group_sum(gx, LPH);
                            }
                            rinv = 1.f / sqrtf(xx / count + A.eps);
                            mean = gx * rinv / count;
                        } else if (h < A.H) {
                            load_weight<D, ADJ>(weight + h * D, c, w);
                        }
                        norm_gradient(vx, vg, w, rinv, mean, acc, DW == DW_STEP && h < A.H);
                    }
                    rg[s] = encode<T>(vg);
                }
                if (h < A.H) store_pairs<T, D, ADJ>(dx + h * A.ds[2], c, rg[s]);
            }
        }
    }

    if (DW == DW_STEP && weight) {              // the same for the whole block
        // lanes of one column: all heads and tokens of the wavefront, or (whole) its tokens
        const int from = whole ? G : LPH, slot = (threadIdx.x & 63) / LPH;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            for (int o = from; o < 64; o <<= 1) acc[k] += __shfl_xor(acc[k], o);
        for (int turn_of = 0; turn_of < 4; ++turn_of) {
            if (wave == turn_of && (whole ? slot < HPS && slot < A.H : slot == 0)) add_to<D, ADJ>(s_dw + (whole ? slot * D : 0), c, acc, wave == 0);
            __syncthreads();
        }
        float *out = A.partial + ((size_t)t * A.P + blockIdx.x) * A.cols;
        for (int i = threadIdx.x; i < A.cols; i += 256) out[i] = s_dw[i];
    }
}

// DW_ROW: grid (P, tensors), block G = 64 or 256: workgroups stride over the tokens, S steps of 8 G values hold one.  The angles of a
// token are formed by its first d/2 threads, one each, and go round through LDS.  Two copies of what goes through LDS, used in turn:
// a copy is written again only behind a barrier that every thread reaches after it has read it.
template <typename T, int D, bool ADJ, int G, int S> __global__ __launch_bounds__(G) void rope_bwd_row_kernel(const RopeArgs A)
{
    constexpr int LPH = D / 8, HPS = G / LPH, WAVES = G / 64;
    __shared__ __attribute__((aligned(16))) float s_cs[2][D / 2], s_sn[2][D / 2];
    __shared__ float s_sum[2][WAVES][2];
    const int tid = threadIdx.x, wave = tid >> 6, t = blockIdx.y, hl = tid / LPH, c = tid % LPH, tokens = A.B * A.N;
    const float *weight = A.weight[t];
    const bool rotate = (A.rotate >> t) & 1;
    float acc[S][8], w[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[s][k] = w[s][k] = 0.f;
        if (weight && s * HPS + hl < A.H) load_weight<D, ADJ>(weight + (s * HPS + hl) * D, c, w[s]);
    }
    int copy = 0;
    for (int token = blockIdx.x; token < tokens; token += gridDim.x, copy ^= 1) {
        const int b = token / A.N, n = token - b * A.N;
        const T *x = static_cast<const T *>(A.src[t]) + b * A.ss[0] + n * A.ss[1];
        const T *g = static_cast<const T *>(A.grad[t]) + b * A.gs[0] + n * A.gs[1];
        T *dx = static_cast<T *>(A.dst[t]) + b * A.ds[0] + n * A.ds[1];
        Raw<T> rg[S], rx[S];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int h = s * HPS + hl;
            if (h >= A.H) continue;
            rg[s] = load_pairs<T, D, ADJ>(g + h * A.gs[2], c);
            if (weight) rx[s] = load_pairs<T, D, ADJ>(x + h * A.ss[2], c);
        }
        float cs[4], sn[4], rinv = 1.f, mean = 0.f;
        if (rotate) {
            if (tid < D / 2) angle(A, position(A, b, n), tid, s_cs[copy][tid], s_sn[copy][tid]);
            __syncthreads();
            const float4 u = *reinterpret_cast<const float4 *>(&s_cs[copy][4 * c]), v = *reinterpret_cast<const float4 *>(&s_sn[copy][4 * c]);
            cs[0] = u.x; cs[1] = u.y; cs[2] = u.z; cs[3] = u.w;
            sn[0] = v.x; sn[1] = v.y; sn[2] = v.z; sn[3] = v.w;
        }
        if (weight) {
            float xx = 0.f, gx = 0.f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                if (s * HPS + hl >= A.H) continue;
                float vx[8], vg[8];
                decode(rx[s], vx);
                decode(rg[s], vg);
                if (rotate) turn<ADJ>(vg, cs, sn, A.sense);
                add_sums(vx, vg, w[s], xx, gx);
            }
            xx = group_sum(xx, 64);
            gx = group_sum(gx, 64);
            if (WAVES > 1) {
                if ((tid & 63) == 0) {
                    s_sum[copy][wave][0] = xx;
                    s_sum[copy][wave][1] = gx;
                }
                __syncthreads();
                xx = gx = 0.f;
#pragma unroll
                for (int k = 0; k < WAVES; ++k) {
                    xx += s_sum[copy][k][0];
                    gx += s_sum[copy][k][1];
                }
            }
            const float count = (float)A.H * D;
            rinv = 1.f / sqrtf(xx / count + A.eps);
            mean = gx * rinv / count;
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int h = s * HPS + hl;
            if (h >= A.H) continue;
            if (weight || rotate) {
                float vg[8];
                decode(rg[s], vg);
                if (rotate) turn<ADJ>(vg, cs, sn, A.sense);
                if (weight) {
                    float vx[8];
                    decode(rx[s], vx);
                    norm_gradient(vx, vg, w[s], rinv, mean, acc[s], true);
                }
                rg[s] = encode<T>(vg);
            }
            store_pairs<T, D, ADJ>(dx + h * A.ds[2], c, rg[s]);
        }
    }
    if (weight) {
        float *out = A.partial + ((size_t)t * A.P + blockIdx.x) * A.cols;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int h = s * HPS + hl;
            if (h >= A.H) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) out[h * D + column<D, ADJ>(c, k)] = acc[s][k];
        }
    }
}

// DW_LONG: grid (ceil(H / HPS), P, tensors), block 256: one step of heads, every P-th group of four tokens
template <typename T, int D, bool ADJ> __global__ __launch_bounds__(256) void rope_dw_long_kernel(const RopeArgs A)
{
    constexpr int LPH = D / 8, HPS = 64 / LPH;
    __shared__ float s_dw[512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = blockIdx.z;
    const int hl = lane / LPH, c = lane % LPH, h = blockIdx.x * HPS + hl, tokens = A.B * A.N;
    if (!A.weight[t]) return;
    const bool rotate = (A.rotate >> t) & 1;
    float acc[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = 0.f;
    for (int token = blockIdx.y * 4 + wave; token < tokens; token += gridDim.y * 4) {
        const int b = token / A.N, n = token - b * A.N;
        float cs[4], sn[4];
        if (rotate) angles(A, b, n, c, cs, sn);
        const float rinv = A.rinv[(size_t)t * tokens + token];
        if (h < A.H) {
            float vx[8], vg[8];
            decode(load_pairs<T, D, ADJ>(static_cast<const T *>(A.src[t]) + b * A.ss[0] + n * A.ss[1] + h * A.ss[2], c), vx);
            decode(load_pairs<T, D, ADJ>(static_cast<const T *>(A.grad[t]) + b * A.gs[0] + n * A.gs[1] + h * A.gs[2], c), vg);
            if (rotate) turn<ADJ>(vg, cs, sn, A.sense);
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] += vg[k] * (vx[k] * rinv);
        }
    }
    for (int turn_of = 0; turn_of < 4; ++turn_of) {
        if (wave == turn_of) add_to<D, ADJ>(s_dw + hl * D, c, acc, wave == 0);
        __syncthreads();
    }
    float *out = A.partial + ((size_t)t * A.P + blockIdx.y) * A.cols + (size_t)blockIdx.x * 512;
    for (int i = threadIdx.x; i < 512; i += 256)
        if ((size_t)blockIdx.x * 512 + i < (size_t)A.cols) out[i] = s_dw[i];
}

// grid (ceil(cols / 64), tensors), block 1024: dw = sum of the P partial sums, 64 bits; 16 wavefronts take every 16th
__global__ __launch_bounds__(1024) void rope_dw_kernel(const RopeArgs A)
{
    __shared__ double s[16][64];
    const int t = blockIdx.y, j = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + j;
    if (!A.weight[t]) return;
    double sum = 0.0;
    if (i < A.cols) {
        const float *p = A.partial + ((size_t)t * A.P + wave) * A.cols + i;
#pragma unroll 8
        for (int k = wave; k < A.P; k += 16, p += 16 * (size_t)A.cols) sum += *p;
    }
    s[wave][j] = sum;
    __syncthreads();
    if (wave == 0 && i < A.cols) {
        for (int k = 1; k < 16; ++k) sum += s[k][j];
        A.dw[t][i] = (float)sum;
    }
}

// ---- launchers -------------------------------------------------------------
static RopeArgs device_args(const svg2_rope_args *a)
{
    RopeArgs A = {};
    for (int t = 0; t < a->n_tensors; ++t) {
        A.src[t] = a->src[t];
        A.dst[t] = a->dst[t];
        A.weight[t] = a->norm_weight[t];
        A.rotate |= a->rotate[t] ? 1 << t : 0;
    }
    for (int k = 0; k < 3; ++k) {
        A.ss[k] = a->src_stride[k];
        A.ds[k] = a->dst_stride[k];
    }
    A.pos = a->pos;
    A.pos_b = a->pos_stride_b;
    A.freq = a->freq;
    A.n_axes = a->n_axes;
    for (int k = 0, e = 0; k < a->n_axes; ++k) A.end[k] = e += a->axis_pairs[k];
    A.B = a->B;
    A.N = a->N;
    A.H = a->H;
    A.token_scope = a->norm_scope == SVG2_NORM_TOKEN;
    A.eps = a->eps;
    A.sense = 1.f;
    return A;
}

template <typename F> static int with_types(const svg2_rope_args *a, F f)
{
    const bool adj = a->pairing == SVG2_ROPE_ADJACENT;
    if (a->dtype == SVG2_BF16) {
        if (a->d == 128) return adj ? f((bf16_t *)0, std::integral_constant<int, 128>(), std::true_type()) : f((bf16_t *)0, std::integral_constant<int, 128>(), std::false_type());
        return adj ? f((bf16_t *)0, std::integral_constant<int, 64>(), std::true_type()) : f((bf16_t *)0, std::integral_constant<int, 64>(), std::false_type());
    }
    if (a->d == 128) return adj ? f((float *)0, std::integral_constant<int, 128>(), std::true_type()) : f((float *)0, std::integral_constant<int, 128>(), std::false_type());
    return adj ? f((float *)0, std::integral_constant<int, 64>(), std::true_type()) : f((float *)0, std::integral_constant<int, 64>(), std::false_type());
}

// f(lanes) with the lanes that take a token of one step, H heads of D: 8 (D = 64), 16, 32 or 64
template <int D, typename F> static void with_lanes(int H, F f)
{
    const int lanes = H * (D / 8);
    if (D == 64 && lanes <= 8) f(std::integral_constant<int, D == 64 ? 8 : 16>());
    else if (lanes <= 16) f(std::integral_constant<int, 16>());
    else if (lanes <= 32) f(std::integral_constant<int, 32>());
    else f(std::integral_constant<int, 64>());
}

// A launch takes fewer than 2^32 threads in a dimension, and 2^26 tokens of a wavefront each are that many: the workgroups behind the
// first 2^23 go into the third dimension.  Some of the last row of them have no token: rope_kernel asks.
static dim3 token_grid(int workgroups, int tensors)
{
    const int most = 1 << 23;
    return workgroups <= most ? dim3(workgroups, tensors) : dim3(most, tensors, cdiv(workgroups, most));
}

static int forward(const svg2_rope_args *a, const RopeArgs &A, hipStream_t st)
{
    return with_types(a, [&](auto *tp, auto dim, auto adj) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        constexpr int D = decltype(dim)::value;
        constexpr bool ADJ = decltype(adj)::value;
        const int lanes = A.H * (D / 8), tokens = A.B * A.N;
        // More than two steps of a wavefront: a workgroup a token, up to where both are bound by memory (figures beside rope_row_kernel).
        // Its edges, us for Q, K and V of heads of 128: 48 heads are the most that rope_row_kernel's three steps hold, one token 3.7, 49
        // heads by a wavefront 9.5; 40 heads are the most that rope_kernel's ten steps hold, a longer token is read twice under a norm over
        // the token: 75,600 tokens of 40 heads 859, of 41 heads 1008 (norm per head, read once: 864 and 897).
        if (lanes > 128 && tokens <= 8192 && lanes <= 256) rope_row_kernel<T, D, ADJ, 1><<<dim3(tokens, a->n_tensors), 256, 0, st>>>(A);
        else if (lanes > 128 && tokens <= 8192 && lanes <= 768) rope_row_kernel<T, D, ADJ, 3><<<dim3(tokens, a->n_tensors), 256, 0, st>>>(A);
        else if (lanes > 128) rope_kernel<T, D, ADJ, 64, 10><<<token_grid(cdiv(tokens, 4), a->n_tensors), 256, 0, st>>>(A);
        else with_lanes<D>(A.H, [&](auto g) {
            constexpr int G = decltype(g)::value;
            rope_kernel<T, D, ADJ, G, G == 64 ? 2 : 1><<<token_grid(cdiv(tokens, 256 / G), a->n_tensors), 256, 0, st>>>(A);
        });
        SVG2_HIP_CHECK(hipGetLastError());
        return SVG2_OK;
    });
}

int rope_launch(const svg2_rope_args *a, hipStream_t st) { return forward(a, device_args(a), st); }

struct RopeBwdPlan {
    int dw, P, blocks, cols, lanes;
    size_t rinv_bytes, total;
};

static RopeBwdPlan bwd_plan(const svg2_rope_args *a)
{
    RopeBwdPlan p = {};
    const int tokens = a->B * a->N;
    bool normed = false;
    for (int t = 0; t < a->n_tensors; ++t) normed |= a->norm_weight[t] != nullptr;
    if (!normed) p.dw = DW_NONE;
    else if (a->norm_scope == SVG2_NORM_HEAD || a->H * a->d <= 512) p.dw = DW_STEP;
    else p.dw = a->H * a->d <= ROW_STEPS * 2048 ? DW_ROW : DW_LONG;
    p.cols = a->norm_scope == SVG2_NORM_HEAD ? a->d : a->H * a->d;
    p.lanes = a->H * (a->d / 8) <= 8 ? 8 : a->H * (a->d / 8) <= 16 ? 16 : a->H * (a->d / 8) <= 32 ? 32 : 64;
    p.blocks = p.dw == DW_ROW ? tokens : cdiv(tokens, p.dw == DW_STEP ? 256 / p.lanes : 4);
    if (p.dw == DW_STEP || p.dw == DW_ROW) {            // one partial sum per block: two blocks of 256 per CU and tensor
        const int most = p.dw == DW_ROW && p.cols <= ROW_STEPS * 512 ? 2048 : 512;
        if (p.blocks > most) p.blocks = most;
        p.P = p.blocks;
    } else if (p.dw == DW_LONG) {                       // 64 slices of the tokens, fewer where a partial sum is long
        const int most = 1 + (1 << 23) / p.cols;
        p.P = p.blocks < 64 ? p.blocks : 64;
        if (p.P > most) p.P = most;
        p.rinv_bytes = align256(3 * (size_t)tokens * sizeof(float));
        if (p.blocks > 1 << 22) p.blocks = 1 << 22;     // its workgroups stride over the tokens (a launch: see token_grid)
    }
    p.total = p.rinv_bytes + 3 * (size_t)p.P * p.cols * sizeof(float);
    if (p.total < 256) p.total = 256;
    return p;
}

size_t rope_bwd_ws_bytes(const svg2_rope_args *a) { return bwd_plan(a).total; }

int rope_bwd_launch(const svg2_rope_args *a, const void *const *dY, void *const *dX, const int64_t *dx_stride,
                    float *const *dW, void *ws, hipStream_t st)
{
    RopeArgs A = device_args(a);
    const RopeBwdPlan p = bwd_plan(a);
    for (int t = 0; t < a->n_tensors; ++t) {
        A.grad[t] = dY[t];
        A.dst[t] = dX[t];
        A.dw[t] = A.weight[t] ? dW[t] : nullptr;
    }
    for (int k = 0; k < 3; ++k) {
        A.gs[k] = a->dst_stride[k];
        A.ds[k] = dx_stride[k];
    }
    A.sense = -1.f;
    if (p.dw == DW_NONE) {
        for (int t = 0; t < a->n_tensors; ++t) A.src[t] = dY[t];
        for (int k = 0; k < 3; ++k) A.ss[k] = a->dst_stride[k];
        return forward(a, A, st);
    }
    A.rinv = static_cast<float *>(ws);
    A.partial = reinterpret_cast<float *>(static_cast<char *>(ws) + p.rinv_bytes);
    A.P = p.P;
    A.cols = p.cols;
    return with_types(a, [&](auto *tp, auto dim, auto adj) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        constexpr int D = decltype(dim)::value;
        constexpr bool ADJ = decltype(adj)::value;
        const dim3 grid(p.blocks, a->n_tensors);
        if (p.dw == DW_STEP) with_lanes<D>(A.H, [&](auto g) { rope_bwd_kernel<T, D, ADJ, DW_STEP, decltype(g)::value><<<grid, 256, 0, st>>>(A); });
        else if (p.dw == DW_LONG) rope_bwd_kernel<T, D, ADJ, DW_LONG, 64><<<grid, 256, 0, st>>>(A);
        else if (p.cols <= 1024) rope_bwd_row_kernel<T, D, ADJ, 64, 2><<<grid, 64, 0, st>>>(A);
        else if (p.cols <= 2048) rope_bwd_row_kernel<T, D, ADJ, 64, 4><<<grid, 64, 0, st>>>(A);
        else if (p.cols <= 4096) rope_bwd_row_kernel<T, D, ADJ, 256, 2><<<grid, 256, 0, st>>>(A);
        else if (p.cols <= 6144) rope_bwd_row_kernel<T, D, ADJ, 256, 3><<<grid, 256, 0, st>>>(A);
        else rope_bwd_row_kernel<T, D, ADJ, 256, 4><<<grid, 256, 0, st>>>(A);
        SVG2_HIP_CHECK(hipGetLastError());
        if (p.dw == DW_LONG) {
            rope_dw_long_kernel<T, D, ADJ><<<dim3(cdiv(p.cols, 512), p.P, a->n_tensors), 256, 0, st>>>(A);
            SVG2_HIP_CHECK(hipGetLastError());
        }
        rope_dw_kernel<<<dim3(cdiv(p.cols, 64), a->n_tensors), 1024, 0, st>>>(A);
        SVG2_HIP_CHECK(hipGetLastError());
        return SVG2_OK;
    });
}

}  // namespace svg2

// Whole rows of activations: to 8 bits with a scale each (quantize_rows_kernel), and what stands between two
// blocks (norm_residual_kernel: the norm behind a block, its gate, the residual's scale and sum, the norm in front of
// the next block).  Both can rotate the row (the random Hadamard transform of Section 2.1 of arXiv 2406.11235) before it
// is stored.
//
// A workgroup has a whole row in registers, in quads of four neighbouring values: every value is read once and written
// once, and means, variances and maxima are taken of registers, each with one exchange through LDS.  While one workgroup
// waits for its row others on the CU work on theirs.  Everything between loads and stores is binary32.
#include "qtip_device.h"
#include "qtip_internal.h"
#include "qtip_rht_device.h"
#include "qtip_rows_device.h"

namespace qtip {

namespace {

// Where a thread's quad number q lies in its row.  Rotated rows: chunks of 4096 by 16 waves, as rht_chunk takes
// (in) and leaves (out) them.
template <bool ROT> __device__ __forceinline__ int quad_in(int q) {
    if constexpr (ROT) return q * RHT_CHUNK + rht_in_index(threadIdx.x >> 6, threadIdx.x & 63);
    else return 4 * (q * (int)blockDim.x + (int)threadIdx.x);
}
template <bool ROT> __device__ __forceinline__ int quad_out(int q) {
    if constexpr (ROT) return q * RHT_CHUNK + rht_out_index(threadIdx.x >> 6, threadIdx.x & 63);
    else return 4 * (q * (int)blockDim.x + (int)threadIdx.x);
}

// v: quads at quad_in() to quads at quad_out() of V (S .* v), blocks of 2^p values.
template <int Q>
__device__ __forceinline__ void rotate_row(float4_t (&v)[Q], const int8_t *__restrict__ signs, int n, int p, float *s_v) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    uint32_t s[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int at = quad_in<true>(q);
        s[q] = at < n ? *reinterpret_cast<const uint32_t *>(signs + at) : 0u;
    }
    RhtMatrix M;
    M.init(lane);
    const float scale = rht_scale(p);
#pragma unroll
    for (int q = 0; q < Q; q++) {
        if (q * RHT_CHUNK >= n) break;
        const float4_t in[1] = {rht_signed(v[q], s[q])};
        float4_t out[1];
        rht_chunk<16>(in, M, p, 16, s_v + (q & 1) * RHT_LDS_FLOATS, wave, lane, out);
        v[q] = out[0];
    }
    // the butterflies between the chunks of blocks of 8192 and 16384
#pragma unroll
    for (int h = 1; h < 4; h <<= 1) {
        if (p < (h == 1 ? 13 : 14)) break;
#pragma unroll
        for (int q = 0; q < Q; q++)
            if ((q & h) == 0 && (q | h) < Q) {
                const float4_t a = v[q], b = v[q | h];
                v[q] = a + b;
                v[q | h] = a - b;
            }
    }
#pragma unroll
    for (int q = 0; q < Q; q++) v[q] *= scale;
}

// The bits of the largest absolute value: they order as whole numbers, NaN above infinity, so one maximum finds those too.
template <int Q, bool ROT> __device__ __forceinline__ uint32_t largest(const float4_t (&v)[Q], int n) {
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < Q; q++)
        if (quad_out<ROT>(q) < n) {
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const float one = v[q][r];
                top = max(top, __builtin_bit_cast(uint32_t, one) & 0x7FFFFFFFu);
            }
        }
    return top;
}
// v to 8 bits: scale = a / 127 and q = v (127 / a) to the nearest whole number, ties to even, a = `top` the row's largest absolute
// value.  A row of zeros has the scale 0; one with an infinity or a NaN has the scale NaN, so that what is computed of it is NaN too.
template <int Q, bool ROT, bool RAGGED>
__device__ __forceinline__ void store_i8(const float4_t (&v)[Q], int n, int8_t *__restrict__ to, float *scale, uint32_t top) {
    const float a = __builtin_bit_cast(float, top);
    const bool finite = top < 0x7F800000u;
    if (threadIdx.x == 0) *scale = finite ? a / 127.f : __builtin_nanf("");
    const float inverse = 127.f / a;
    // (127 / a overflows below 2^-121, and is 127 / 0 for a row of zeros)
    const bool plain = finite && a >= 0x1p-120f;
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int at = quad_out<ROT>(q);
        if (at >= n) continue;
        uint32_t word = 0;
        if (plain) {
            // v (127 / a), at most 127 large, and 1.5 2^23: the sum's last 8 bits are the nearest whole number's
            uint32_t b[4];
#pragma unroll
            for (int r = 0; r < 4; r++) {
                float t = v[q][r] * inverse;
                asm("" : "+v"(t));  // (a rounding of its own: not a fused product and sum)
                b[r] = __builtin_bit_cast(uint32_t, t + 12582912.f);
            }
            word = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0C0C0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), 0x05040100u);
        } else if (finite && top) {
#pragma unroll
            for (int r = 0; r < 4; r++) word |= ((uint32_t)(int)__builtin_rintf(v[q][r] / a * 127.f) & 0xFFu) << (8 * r);
        }
        store_quad<RAGGED>(to, at, n, word);
    }
}

template <int Q, bool ROT, bool RAGGED>
__device__ __forceinline__ void store_row(const float4_t (&v)[Q], int n, int type, void *x, int64_t at_row) {
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int at = quad_out<ROT>(q);
        if (type == TYPE_F32) store_quad<RAGGED>((float *)x + at_row, at, n, v[q]);
        else if (type == TYPE_F16) store_quad<RAGGED>((half_t *)x + at_row, at, n, v[q]);
        else store_quad<RAGGED>((bf16_t *)x + at_row, at, n, v[q]);
    }
}

constexpr int rotate_lds(bool rot) { return rot ? 2 * RHT_LDS_FLOATS : 1; }

template <class T, int Q, bool ROT, bool RAGGED> __device__ __forceinline__ void load_row(typename Quad<T>::type (&v)[Q], const T *row, int n) {
#pragma unroll
    for (int q = 0; q < Q; q++) v[q] = load_quad<RAGGED>(row, quad_in<ROT>(q), n);
}
template <class T, int Q, bool ROT, bool RAGGED>
__global__ __launch_bounds__(1024) void quantize_rows_kernel(const T *__restrict__ x, const T *__restrict__ up, int n, int64_t ldx,
                                                             const int8_t *__restrict__ signs, int p, int8_t *__restrict__ out,
                                                             int64_t ldq, float *__restrict__ scale) {
    __shared__ __attribute__((aligned(16))) float s_v[rotate_lds(ROT)];
    __shared__ uint32_t s_max[16];
    const int64_t row = blockIdx.x;
    typename Quad<T>::type raw[Q], raw_up[Q];
    load_row<T, Q, ROT, RAGGED>(raw, x + row * ldx, n);
    if (up) load_row<T, Q, ROT, RAGGED>(raw_up, up + row * ldx, n);
    float4_t v[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        v[q] = widen(raw[q]);
        if (up) {
            const float4_t u = widen(raw_up[q]);
#pragma unroll
            for (int r = 0; r < 4; r++) v[q][r] = silu(v[q][r]) * u[r];
        }
    }
    if constexpr (ROT) rotate_row<Q>(v, signs, n, p, s_v);
    const uint32_t top = block_max(largest<Q, ROT>(v, n), s_max, blockDim.x >> 6);
    store_i8<Q, ROT, RAGGED>(v, n, out + row * ldq, scale + row, top);
}

// v: (v - mean) / sqrt(mean of (v - mean)^2 + eps) * weight + bias; the mean is 0 where the norm has none.  Zeros beyond n stay.
template <int Q, bool ROT>
__device__ __forceinline__ void normalize(float4_t (&v)[Q], int n, float over_n, bool layer, float eps, float (*slots)[16], int waves) {
    if (layer) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < Q; q++) t += (v[q][0] + v[q][1]) + (v[q][2] + v[q][3]);
        const float mean = block_sum(t, slots[0], waves) * over_n;
#pragma unroll
        for (int q = 0; q < Q; q++)
#pragma unroll
            for (int r = 0; r < 4; r++) v[q][r] = quad_in<ROT>(q) + r < n ? v[q][r] - mean : 0.f;
    }
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < Q; q++) t += (v[q][0] * v[q][0] + v[q][1] * v[q][1]) + (v[q][2] * v[q][2] + v[q][3] * v[q][3]);
    const float scale = 1.f / __builtin_sqrtf(block_sum(t, slots[1], waves) * over_n + eps);
#pragma unroll
    for (int q = 0; q < Q; q++) v[q] *= scale;
}

template <class TY, class TH, int Q, bool ROT, bool RAGGED>
__global__ __launch_bounds__(1024) void norm_residual_kernel(NormResidual a) {
    __shared__ __attribute__((aligned(16))) float s_v[rotate_lds(ROT)];
    __shared__ float s_sum[4][16];
    __shared__ uint32_t s_max[16];
    const int64_t row = blockIdx.x;
    const int n = a.n, waves = blockDim.x >> 6;
    const float over_n = 1.f / (float)n;
    typename Quad<TY>::type y[Q], g[Q];
    typename Quad<TH>::type h[Q];
    if (a.y) load_row<TY, Q, ROT, RAGGED>(y, (const TY *)a.y + row * a.ldy, n);
    if (a.h) load_row<TH, Q, ROT, RAGGED>(h, (const TH *)a.h + row * a.ldh, n);
    if (a.gate) load_row<TY, Q, ROT, RAGGED>(g, (const TY *)a.gate + row * a.ldgate, n);
    float4_t v[Q];
    auto affine = [&](const float *weight, const float *bias) {
#pragma unroll
        for (int q = 0; q < Q; q++) {
            v[q] *= load_quad<RAGGED>(weight, quad_in<ROT>(q), n);
            if (bias) v[q] += load_quad<RAGGED>(bias, quad_in<ROT>(q), n);
        }
    };
#pragma unroll
    for (int q = 0; q < Q; q++) v[q] = a.y ? widen(y[q]) : widen(h[q]);
    if (a.post) {
        normalize<Q, ROT>(v, n, over_n, a.layer, a.eps, s_sum, waves);
        affine(a.post, a.post_bias);
    }
    if (a.y) {
#pragma unroll
        for (int q = 0; q < Q; q++) {
            if (a.gate) v[q] *= widen(g[q]);
            v[q] *= a.res_scale;
            if (a.h) v[q] += widen(h[q]);
        }
    }
    if (a.h_out) {
#pragma unroll
        for (int q = 0; q < Q; q++) store_quad<RAGGED>((TH *)a.h_out + row * a.ldh, quad_in<ROT>(q), n, v[q]);
    }
    if (!a.x) return;
    if (a.pre) {
        normalize<Q, ROT>(v, n, over_n, a.layer, a.eps, s_sum + 2, waves);
        affine(a.pre, a.pre_bias);
    }
    if constexpr (ROT) rotate_row<Q>(v, a.signs, n, a.p, s_v);
    if (a.x_type == TYPE_I8) {
        const uint32_t top = block_max(largest<Q, ROT>(v, n), s_max, waves);
        store_i8<Q, ROT, RAGGED>(v, n, (int8_t *)a.x + row * a.ldx, a.x_scale + row, top);
    } else {
        store_row<Q, ROT, RAGGED>(v, n, a.x_type, a.x, row * a.ldx);
    }
}

int log2_of(int block) {
    int p = 0;
    while ((1 << p) < block) p++;
    return p;
}

}  // namespace

// Quads of a thread, then as many waves as hold the row.  One quad while there is at most a row for each CU (the shortest way
// from load to store), else four: more rows on a CU at a time (us, one, two, four, eight quads: norms 4096 x 8192 67.4, 67.4, 65.4,
// 108; 997 x 5003 20.5, 20.4, 17.0, 26.0; 4096 x 4096 33.3, 26.9, 27.4, 39.1; to 8 bits 4096 x 4096 13.6, 10.7, 10.6, 10.3).
// Rotated rows: 16 waves and whole chunks of 4096.
struct Shape {
    int quads, waves;
};
static Shape shape_of(int rows, int n, bool rot) {
    if (rot) return {n <= 4096 ? 1 : n <= 8192 ? 2 : n <= 16384 ? 4 : 8, 16};
    int quads = rows <= CUS ? 1 : 4;
    while (n > 4096 * quads) quads *= 2;
    return {quads, (n + 256 * quads - 1) / (256 * quads)};
}
#define QTIP_ROWS_BY_QUADS(LAUNCH, s, rot, ragged)  \
    if (s.quads == 1) LAUNCH(1, rot, ragged);       \
    else if (s.quads == 2) LAUNCH(2, rot, ragged);  \
    else if (s.quads == 4) LAUNCH(4, rot, ragged);  \
    else LAUNCH(8, rot, ragged)
#define QTIP_ROWS_BY_SHAPE(LAUNCH, s, n, rot)                         \
    if (rot) { QTIP_ROWS_BY_QUADS(LAUNCH, s, true, false); }          \
    else if (n % 4) { QTIP_ROWS_BY_QUADS(LAUNCH, s, false, true); }   \
    else { QTIP_ROWS_BY_QUADS(LAUNCH, s, false, false); }

template <class T>
static void launch_quantize(const void *x, const void *up, int rows, int n, int64_t ldx, const int8_t *signs, int p, int8_t *q,
                            int64_t ldq, float *scale, hipStream_t st) {
    const Shape s = shape_of(rows, n, signs);
#define QTIP_QUANTIZE(Q, ROT, RAGGED)                                                                                                 \
    hipLaunchKernelGGL((quantize_rows_kernel<T, Q, ROT, RAGGED>), dim3(rows), dim3(s.waves * 64), 0, st, (const T *)x, (const T *)up, n, \
                       ldx, signs, p, q, ldq, scale)
    QTIP_ROWS_BY_SHAPE(QTIP_QUANTIZE, s, n, signs);
}

hipError_t launch_quantize_rows_i8(const void *x, const void *up, int type, int rows, int n, int64_t ldx, const int8_t *signs,
                                   int block, int8_t *q, int64_t ldq, float *scale, hipStream_t st) {
    const int p = signs ? log2_of(block) : 0;
    if (type == TYPE_F32) launch_quantize<float>(x, up, rows, n, ldx, signs, p, q, ldq, scale, st);
    else if (type == TYPE_F16) launch_quantize<half_t>(x, up, rows, n, ldx, signs, p, q, ldq, scale, st);
    else launch_quantize<bf16_t>(x, up, rows, n, ldx, signs, p, q, ldq, scale, st);
    return hipGetLastError();
}

template <class TY, class TH> static void launch_norm(const NormResidual &a, int rows, hipStream_t st) {
    const Shape s = shape_of(rows, a.n, a.signs);
#define QTIP_NORM(Q, ROT, RAGGED) \
    hipLaunchKernelGGL((norm_residual_kernel<TY, TH, Q, ROT, RAGGED>), dim3(rows), dim3(s.waves * 64), 0, st, a)
    QTIP_ROWS_BY_SHAPE(QTIP_NORM, s, a.n, a.signs);
}

hipError_t launch_norm_residual(NormResidual a, int y_type, int h_type, int rows, int block, hipStream_t st) {
    a.p = a.signs ? log2_of(block) : 0;
    if (y_type == TYPE_F32) launch_norm<float, float>(a, rows, st);
    else if (y_type == TYPE_F16) h_type == TYPE_F32 ? launch_norm<half_t, float>(a, rows, st) : launch_norm<half_t, half_t>(a, rows, st);
    else h_type == TYPE_F32 ? launch_norm<bf16_t, float>(a, rows, st) : launch_norm<bf16_t, bf16_t>(a, rows, st);
    return hipGetLastError();
}

}  // namespace qtip

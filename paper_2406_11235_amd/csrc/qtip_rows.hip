// Whole rows of activations: to 8 bits with a scale each (quantize_rows_kernel), and what stands between two
// blocks (norm_residual_kernel: the norm behind a block, its gate, the residual's scale and sum, the norm in front of
// the next block).  Both can rotate the row (the random Hadamard transform of Section 2.1 of arXiv 2406.11235) before it
// is stored.
//
// A workgroup has a whole row in registers, in quads of four neighbouring values: every value is read once and written
// once, and means, variances and maxima are taken of registers, each with one exchange through LDS.  Everything
// between loads and stores is binary32.
#include "qtip_device.h"
#include "qtip_internal.h"
#include "qtip_rht_device.h"
#include "qtip_rows_device.h"

namespace qtip {

namespace {

// Where a thread's quad number q lies in its row.  Rotated rows: chunks of 4096 by 16 waves, as rht_chunk takes
// (in) and leaves (out) them.
template <int NW, bool ROT> __device__ __forceinline__ int quad_in(int q) {
    if constexpr (ROT) return q * RHT_CHUNK + rht_in_index(threadIdx.x >> 6, threadIdx.x & 63);
    else return 4 * (q * NW * 64 + (int)threadIdx.x);
}
template <int NW, bool ROT> __device__ __forceinline__ int quad_out(int q) {
    if constexpr (ROT) return q * RHT_CHUNK + rht_out_index(threadIdx.x >> 6, threadIdx.x & 63);
    else return 4 * (q * NW * 64 + (int)threadIdx.x);
}

// v: quads at quad_in() to quads at quad_out() of V (S .* v), blocks of 2^p values.
template <int Q>
__device__ __forceinline__ void rotate_row(float4_t (&v)[Q], const int8_t *__restrict__ signs, int n, int p, float *s_v) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    uint32_t s[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int at = quad_in<16, true>(q);
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

// v to 8 bits: scale = a / 127 and q = v (127 / a) to the nearest whole number, ties to even, a the row's largest absolute value.
// A row of zeros has the scale 0; one with an infinity or a NaN has the scale NaN, so that what is computed of it is NaN too.
template <int NW, int Q, bool ROT>
__device__ __forceinline__ void store_i8(const float4_t (&v)[Q], int n, int8_t *__restrict__ to, float *scale, uint32_t *s_max) {
    // (absolute values order as whole numbers, NaN above infinity: one maximum finds them too)
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < Q; q++)
        if (quad_out<NW, ROT>(q) < n) {
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const float one = v[q][r];
                top = max(top, __builtin_bit_cast(uint32_t, one) & 0x7FFFFFFFu);
            }
        }
    top = block_max<NW>(top, s_max);
    const float a = __builtin_bit_cast(float, top);
    const bool finite = top < 0x7F800000u;
    if (threadIdx.x == 0) *scale = finite ? a / 127.f : __builtin_nanf("");
    const float inverse = 127.f / a;
    // 127 / a overflows below 2^-121 and is 127 / 0 for a row of zeros
    const bool tiny = a < 0x1p-120f;
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int at = quad_out<NW, ROT>(q);
        if (at >= n) continue;
        uint32_t word = 0;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            float t = v[q][r] * inverse;
            if (tiny) t = top ? v[q][r] / a * 127.f : 0.f;
            const int whole = finite ? (int)__builtin_rintf(t) : 0;
            word |= ((uint32_t)whole & 0xFFu) << (8 * r);
        }
        store_quad(to, at, n, word);
    }
}

template <int NW, int Q, bool ROT>
__device__ __forceinline__ void store_row(const float4_t (&v)[Q], int n, int type, void *x, int64_t at_row, float *scale,
                                          uint32_t *s_max) {
    if (type == TYPE_I8) {
        store_i8<NW, Q, ROT>(v, n, (int8_t *)x + at_row, scale, s_max);
        return;
    }
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int at = quad_out<NW, ROT>(q);
        if (type == TYPE_F32) store_quad((float *)x + at_row, at, n, v[q]);
        else if (type == TYPE_F16) store_quad((half_t *)x + at_row, at, n, v[q]);
        else store_quad((bf16_t *)x + at_row, at, n, v[q]);
    }
}

constexpr int rotate_lds(bool rot) { return rot ? 2 * RHT_LDS_FLOATS : 1; }

template <class T, int NW, int Q, bool ROT>
__global__ __launch_bounds__(NW * 64) void quantize_rows_kernel(const T *__restrict__ x, const T *__restrict__ up, int n, int64_t ldx,
                                                                const int8_t *__restrict__ signs, int p,
                                                                int8_t *__restrict__ out, int64_t ldq,
                                                                float *__restrict__ scale) {
    __shared__ __attribute__((aligned(16))) float s_v[rotate_lds(ROT)];
    __shared__ uint32_t s_max[NW];
    const int64_t row = blockIdx.x;
    x += row * ldx;
    typename Quad<T>::type raw[Q], raw_up[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) raw[q] = load_quad(x, quad_in<NW, ROT>(q), n);
    if (up) {
        up += row * ldx;
#pragma unroll
        for (int q = 0; q < Q; q++) raw_up[q] = load_quad(up, quad_in<NW, ROT>(q), n);
    }
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
    store_i8<NW, Q, ROT>(v, n, out + row * ldq, scale + row, s_max);
}

template <class TY, class TH, int NW, int Q, bool ROT>
__global__ __launch_bounds__(NW * 64) void norm_residual_kernel(NormResidual a) {
    __shared__ __attribute__((aligned(16))) float s_v[rotate_lds(ROT)];
    __shared__ __attribute__((aligned(16))) float s_sum[4][NW];
    __shared__ uint32_t s_max[NW];
    const int64_t row = blockIdx.x;
    const int n = a.n;
    const float over_n = 1.f / (float)n;
    typename Quad<TY>::type y[Q], g[Q];
    typename Quad<TH>::type h[Q];
    if (a.y) {
#pragma unroll
        for (int q = 0; q < Q; q++) y[q] = load_quad((const TY *)a.y + row * a.ldy, quad_in<NW, ROT>(q), n);
    }
    if (a.h) {
#pragma unroll
        for (int q = 0; q < Q; q++) h[q] = load_quad((const TH *)a.h + row * a.ldh, quad_in<NW, ROT>(q), n);
    }
    if (a.gate) {
#pragma unroll
        for (int q = 0; q < Q; q++) g[q] = load_quad((const TY *)a.gate + row * a.ldgate, quad_in<NW, ROT>(q), n);
    }
    // (v - mean) / sqrt(mean of (v - mean)^2 + eps) * weight + bias; mean is 0 where the norm has none
    auto normalize = [&](float4_t(&v)[Q], const float *weight, const float *bias, float(*sums)[NW]) {
        float mean = 0.f;
        if (a.layer) {
            float t = 0.f;
#pragma unroll
            for (int q = 0; q < Q; q++) t += (v[q][0] + v[q][1]) + (v[q][2] + v[q][3]);  // (zeros beyond n)
            mean = block_sum<NW>(t, sums[0]) * over_n;
        }
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < Q; q++)
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (quad_in<NW, ROT>(q) + r < n) {
                    v[q][r] -= mean;
                    t += v[q][r] * v[q][r];
                }
        const float scale = 1.f / __builtin_sqrtf(block_sum<NW>(t, sums[1]) * over_n + a.eps);
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const float4_t w = load_quad(weight, quad_in<NW, ROT>(q), n);
            v[q] = v[q] * scale * w;
            if (bias) v[q] += load_quad(bias, quad_in<NW, ROT>(q), n);
        }
    };
    float4_t v[Q];
    if (a.y) {
#pragma unroll
        for (int q = 0; q < Q; q++) v[q] = widen(y[q]);
        if (a.post) normalize(v, a.post, a.post_bias, s_sum);
        if (a.gate) {
#pragma unroll
            for (int q = 0; q < Q; q++) v[q] *= widen(g[q]);
        }
#pragma unroll
        for (int q = 0; q < Q; q++) v[q] *= a.res_scale;
        if (a.h) {
#pragma unroll
            for (int q = 0; q < Q; q++) v[q] += widen(h[q]);
        }
    } else {
#pragma unroll
        for (int q = 0; q < Q; q++) v[q] = widen(h[q]);
    }
    if (a.h_out) {
#pragma unroll
        for (int q = 0; q < Q; q++) store_quad((TH *)a.h_out + row * a.ldh, quad_in<NW, ROT>(q), n, v[q]);
    }
    if (!a.x) return;
    if (a.pre) normalize(v, a.pre, a.pre_bias, s_sum + 2);
    if constexpr (ROT) rotate_row<Q>(v, a.signs, n, a.p, s_v);
    store_row<NW, Q, ROT>(v, n, a.x_type, a.x, row * a.ldx, a.x_scale + row, s_max);
}

int log2_of(int block) {
    int p = 0;
    while ((1 << p) < block) p++;
    return p;
}

}  // namespace

// Waves and quads by the row's length: 16 values a thread where 4 waves hold the row so, else 16 waves.
#define QTIP_ROWS_BY_LENGTH(LAUNCH, n, rot) \
    if (rot) {                              \
        if (n <= 4096) LAUNCH(16, 1, true); \
        else if (n <= 8192) LAUNCH(16, 2, true); \
        else if (n <= 16384) LAUNCH(16, 4, true); \
        else LAUNCH(16, 8, true);           \
    } else if (n <= 1024) LAUNCH(4, 1, false); \
    else if (n <= 2048) LAUNCH(4, 2, false); \
    else if (n <= 4096) LAUNCH(4, 4, false); \
    else if (n <= 8192) LAUNCH(16, 2, false); \
    else if (n <= 16384) LAUNCH(16, 4, false); \
    else LAUNCH(16, 8, false)

hipError_t launch_quantize_rows_i8(const void *x, const void *up, int type, int rows, int n, int64_t ldx, const int8_t *signs,
                                   int block, int8_t *q, int64_t ldq, float *scale, hipStream_t st) {
    const int p = signs ? log2_of(block) : 0;
#define QTIP_QUANTIZE(NW, Q, ROT)                                                                                       \
    do {                                                                                                                \
        if (type == TYPE_F32)                                                                                           \
            hipLaunchKernelGGL((quantize_rows_kernel<float, NW, Q, ROT>), dim3(rows), dim3(NW * 64), 0, st,             \
                               (const float *)x, (const float *)up, n, ldx, signs, p, q, ldq, scale);                   \
        else if (type == TYPE_F16)                                                                                      \
            hipLaunchKernelGGL((quantize_rows_kernel<half_t, NW, Q, ROT>), dim3(rows), dim3(NW * 64), 0, st,            \
                               (const half_t *)x, (const half_t *)up, n, ldx, signs, p, q, ldq, scale);                 \
        else                                                                                                            \
            hipLaunchKernelGGL((quantize_rows_kernel<bf16_t, NW, Q, ROT>), dim3(rows), dim3(NW * 64), 0, st,            \
                               (const bf16_t *)x, (const bf16_t *)up, n, ldx, signs, p, q, ldq, scale);                 \
    } while (0)
    QTIP_ROWS_BY_LENGTH(QTIP_QUANTIZE, n, signs);
    return hipGetLastError();
}

template <class TY, class TH> static void launch_norm(const NormResidual &a, int rows, hipStream_t st) {
#define QTIP_NORM(NW, Q, ROT) \
    hipLaunchKernelGGL((norm_residual_kernel<TY, TH, NW, Q, ROT>), dim3(rows), dim3(NW * 64), 0, st, a)
    QTIP_ROWS_BY_LENGTH(QTIP_NORM, a.n, a.signs);
}

hipError_t launch_norm_residual(NormResidual a, int y_type, int h_type, int rows, int block, hipStream_t st) {
    a.p = a.signs ? log2_of(block) : 0;
    if (y_type == TYPE_F32) launch_norm<float, float>(a, rows, st);
    else if (y_type == TYPE_F16) h_type == TYPE_F32 ? launch_norm<half_t, float>(a, rows, st) : launch_norm<half_t, half_t>(a, rows, st);
    else h_type == TYPE_F32 ? launch_norm<bf16_t, float>(a, rows, st) : launch_norm<bf16_t, bf16_t>(a, rows, st);
    return hipGetLastError();
}

}  // namespace qtip

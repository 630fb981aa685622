// The product of 8-bit rows with 8-bit weights: Y[b][i] = w_scale[i] x_scale[b] sum_j W[i][j] X[b][j] + bias[i], the sum
// exact in 32-bit whole numbers.
#include "qtip_device.h"
#include "qtip_internal.h"
#include "qtip_rows_device.h"

namespace qtip {

namespace {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes at position k of a row of n; what stands behind the row's end is taken as zeros.
__device__ __forceinline__ i32x4_t load_units(const int8_t *row, int k, int n) {
    i32x4_t v = {0, 0, 0, 0};
    if (k < n) v = *reinterpret_cast<const i32x4_t *>(row + k);
    if (k + 16 > n) {
#pragma unroll
        for (int d = 0; d < 4; d++) {
            const int left = n - k - 4 * d;  // bytes of this word that belong to the row
            if (left < 4) v[d] = left <= 0 ? 0 : v[d] & (int)(0xFFFFFFFFu >> (32 - 8 * left));
        }
    }
    return v;
}

// Four neighbouring outputs of batch row b.
template <class T>
__device__ __forceinline__ void store_outputs(const MatmulI8 &a, int b, int i, i32x4_t sum) {
    const float xs = a.x_scale[b];
    float4_t v;
#pragma unroll
    for (int r = 0; r < 4; r++) {
        const int at = min(i + r, a.m - 1);
        v[r] = (float)sum[r] * (a.w_scale[at] * xs) + (a.bias ? a.bias[at] : 0.f);
    }
    store_quad((T *)a.Y + (int64_t)b * a.ldy, i, a.m, v);
}

// 16 outputs x 16 batch rows by a workgroup; its waves take 128 inputs in turn.
template <class T, int NW> __global__ __launch_bounds__(NW * 64) void matmul_i8_few_kernel(MatmulI8 a) {
    __shared__ i32x4_t s_sum[NW][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int i0 = blockIdx.x * 16, b0 = blockIdx.y * 16;
    const int8_t *w = a.W + (int64_t)min(i0 + (lane & 15), a.m - 1) * a.ldw;
    const int8_t *x = a.X + (int64_t)min(b0 + (lane & 15), a.B - 1) * a.ldx;
    i32x4_t sum = {0, 0, 0, 0};
    for (int c = wave * 128; c < a.n; c += NW * 128) {
        const int k = c + 32 * (lane >> 4);
        // (weights behind the row's end meet zeros of x)
        const i32x4_t w0 = load_units(w, k, a.n), w1 = load_units(w, k + 16, a.n);
        const i32x4_t x0 = load_units(x, k, a.n), x1 = load_units(x, k + 16, a.n);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(w0, x0, sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(w1, x1, sum, 0, 0, 0);
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int other = 1; other < NW; other++) sum += s_sum[other][lane];
    const int b = b0 + (lane & 15), i = i0 + 4 * (lane >> 4);
    if (b < a.B && i < a.m) store_outputs<T>(a, b, i, sum);
}

}  // namespace

size_t matmul_i8_workspace(int, int, int) { return 0; }

hipError_t launch_matmul_i8(const MatmulI8 &a, void *, hipStream_t st) {
    const dim3 grid((a.m + 15) / 16, (a.B + 15) / 16);
    if (a.y_type == TYPE_F32) hipLaunchKernelGGL((matmul_i8_few_kernel<float, 4>), grid, dim3(256), 0, st, a);
    else if (a.y_type == TYPE_F16) hipLaunchKernelGGL((matmul_i8_few_kernel<half_t, 4>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((matmul_i8_few_kernel<bf16_t, 4>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qtip

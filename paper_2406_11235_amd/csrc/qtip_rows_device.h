// Quads of four neighbouring values of a row in the types that rows come in, and sums and maxima over a workgroup.
#pragma once
#include "qtip_device.h"

namespace qtip {

typedef __bf16 bf16_t;
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// The vector of four, and the same at any address of an element: rows of odd lengths are read four
// values at a time too (global memory takes vector accesses at any byte).
template <class T> struct Quad {
    typedef T type __attribute__((ext_vector_type(4)));
    typedef T anywhere __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};

__device__ __forceinline__ float4_t widen(float4_t v) { return v; }
__device__ __forceinline__ float4_t widen(half4_t v) { return __builtin_convertvector(v, float4_t); }
__device__ __forceinline__ float4_t widen(bf16x4_t v) { return __builtin_convertvector(v, float4_t); }

// Values at ... at + 3 of a row of n; zeros beyond its end.
template <class T> __device__ __forceinline__ typename Quad<T>::type load_quad(const T *row, int at, int n) {
    typename Quad<T>::type v = {(T)0.f, (T)0.f, (T)0.f, (T)0.f};
    if (at + 4 <= n) {
        v = *reinterpret_cast<const typename Quad<T>::anywhere *>(row + at);
    } else if (at < n) {
        v[0] = row[at];
        if (at + 1 < n) v[1] = row[at + 1];
        if (at + 2 < n) v[2] = row[at + 2];
    }
    return v;
}
template <class T> __device__ __forceinline__ void store_quad(T *row, int at, int n, float4_t v) {
    const typename Quad<T>::type r = __builtin_convertvector(v, typename Quad<T>::type);
    if (at + 4 <= n) {
        *reinterpret_cast<typename Quad<T>::anywhere *>(row + at) = r;
    } else if (at < n) {
        row[at] = r[0];
        if (at + 1 < n) row[at + 1] = r[1];
        if (at + 2 < n) row[at + 2] = r[2];
    }
}
// Four bytes in a word, the first one lowest.
__device__ __forceinline__ void store_quad(int8_t *row, int at, int n, uint32_t word) {
    typedef uint32_t anywhere __attribute__((aligned(1)));
    if (at + 4 <= n) {
        *reinterpret_cast<anywhere *>(row + at) = word;
    } else {
        for (int r = 0; at + r < n; r++) row[at + r] = (int8_t)(word >> (8 * r));
    }
}

__device__ __forceinline__ float silu(float v) { return v / (1.f + __expf(-v)); }

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
// Over the 16 lanes of a row by exchanges with lanes l ^ 1, l ^ 2, l ^ 7 and l ^ 15, then over the four rows: every lane has it.
__device__ __forceinline__ float wave_sum(float v) {
    auto add = [&](uint32_t o) { v += __builtin_bit_cast(float, o); };
    add(dpp<0xB1>(__builtin_bit_cast(uint32_t, v)));
    add(dpp<0x4E>(__builtin_bit_cast(uint32_t, v)));
    add(dpp<0x141>(__builtin_bit_cast(uint32_t, v)));
    add(dpp<0x140>(__builtin_bit_cast(uint32_t, v)));
    const int w = __builtin_bit_cast(int, v);
    auto row = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(w, lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, dpp<0xB1>(v));
    v = max(v, dpp<0x4E>(v));
    v = max(v, dpp<0x141>(v));
    v = max(v, dpp<0x140>(v));
    auto row = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); };
    return max(max(row(0), row(16)), max(row(32), row(48)));
}
// Over NW waves; `slots` is used by no other exchange of the kernel.
template <int NW> __device__ __forceinline__ float block_sum(float v, float *slots) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < NW; w++) t += slots[w];
    return t;
}
template <int NW> __device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *slots) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < NW; w++) t = max(t, slots[w]);
    return t;
}

}  // namespace qtip

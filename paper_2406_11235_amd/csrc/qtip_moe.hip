// A mixture-of-experts layer for a few tokens.  For each token x:
//   l = R x + bias;  the top_k largest l, ties to the lowest expert;  p = softmax(l), over all experts or the chosen ones;
//   h_e = silu(G_e x) .* (U_e x);  y = sum over the chosen e of p_e D_e h_e
// with the experts' weights in 8 bits, a scale for each row, and activations in 16 bits.
//
// What bounds it is reading the chosen experts' weights, once each.  Five launches: logits; the choice; G, U and h; D; the
// sums.  The products run on the matrix cores with 16 rows of weights as one operand and 16 rows of activations as the other;
// weights become 16-bit floats on the way, exactly.  h lives in memory as the sum of two bf16 numbers (16 bits of mantissa at
// any size), two rows of activations for D, so that y is what binary32 would give before its one rounding.
#include <type_traits>

#include "qtip_copy_device.h"
#include "qtip_internal.h"
#include "qtip_rows_device.h"

namespace qtip {

namespace {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// What the choice leaves for the products, in the workspace.
struct Plan {
    int experts;                               // that any token chose, ascending in expert[]
    int expert[MOE_MAX_EXPERTS];
    int first[MOE_MAX_EXPERTS];                // its first pair (a token that chose it); pairs ascend by token
    uint64_t tokens[MOE_MAX_EXPERTS];          // one bit for each token
    float weight[MOE_MAX_TOKENS * MOE_MAX_TOP_K];  // by token and choice
    int token[MOE_MAX_TOKENS * MOE_MAX_TOP_K];
    int pair[MOE_MAX_TOKENS * MOE_MAX_TOP_K];  // by token and choice; -1: left out
};

constexpr size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

struct Workspace {
    Plan *plan;
    float *logits;  // T x E
    bf16_t *h;      // pairs x 2 x f: a row of h rounded, and one of what that left
    float *parts;   // pairs x n: D h
    static size_t bytes(int T, int n, int f, int E, int top_k) {
        return round_up(sizeof(Plan)) + round_up((size_t)T * E * 4) + round_up((size_t)T * top_k * f * 4) + round_up((size_t)T * top_k * n * 4);
    }
    Workspace(void *at, const MoeI8 &a) {
        char *p = (char *)at;
        plan = (Plan *)p;
        p += round_up(sizeof(Plan));
        logits = (float *)p;
        p += round_up((size_t)a.T * a.E * 4);
        h = (bf16_t *)p;
        p += round_up((size_t)a.T * a.top_k * a.f * 4);
        parts = (float *)p;
    }
};

// A wave: the logits of one expert for up to four tokens.
template <class T> __global__ __launch_bounds__(256) void moe_logits_kernel(MoeI8 a, float *__restrict__ logits) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int e = blockIdx.x * 4 + wave, t0 = blockIdx.y * 4;
    if (e >= a.E) return;
    const T *r = (const T *)a.router + (int64_t)e * a.n;
    const T *x[4];
#pragma unroll
    for (int t = 0; t < 4; t++) x[t] = (const T *)a.x + (int64_t)min(t0 + t, a.T - 1) * a.ldx;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 4 * lane; k < a.n; k += 256) {
        const float4_t w = widen(load_quad(r, k, a.n));
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const float4_t v = widen(load_quad(x[t], k, a.n));
            sum[t] += (w[0] * v[0] + w[1] * v[1]) + (w[2] * v[2] + w[3] * v[3]);
        }
    }
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const float l = wave_sum(sum[t]);
        if (lane == 0 && t0 + t < a.T) logits[(t0 + t) * a.E + e] = l + (a.router_bias ? a.router_bias[e] : 0.f);
    }
}

// One workgroup of 16 waves: each takes tokens in turn.
__global__ __launch_bounds__(1024) void moe_choose_kernel(MoeI8 a, Workspace ws) {
    __shared__ unsigned long long s_tokens[MOE_MAX_EXPERTS];
    __shared__ int s_first[MOE_MAX_EXPERTS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (threadIdx.x < MOE_MAX_EXPERTS) s_tokens[threadIdx.x] = 0;
    __syncthreads();
    // of the wave's tokens wave, wave + 16, ...: lane i has the i-th choice
    constexpr int MINE = MOE_MAX_TOKENS / 16;
    int my_id[MINE];
    float my_weight[MINE];
#pragma unroll
    for (int m = 0; m < MINE; m++) {
        const int t = wave + 16 * m;
        my_id[m] = 0;
        my_weight[m] = 0.f;
        if (t >= a.T) break;
        // logits as whole numbers of the same order: NaN below everything, 0 for what is taken or not there
        float l[MOE_MAX_EXPERTS / 64];
        uint32_t key[MOE_MAX_EXPERTS / 64], best = 0;
        bool nan = false;
#pragma unroll
        for (int i = 0; i < MOE_MAX_EXPERTS / 64; i++) {
            const int e = 64 * i + lane;
            l[i] = e < a.E ? ws.logits[t * a.E + e] : -__builtin_inff();
            const uint32_t bits = __builtin_bit_cast(uint32_t, l[i]);
            key[i] = e >= a.E ? 0u : l[i] != l[i] ? 1u : bits & 0x80000000u ? ~bits : bits | 0x80000000u;
            nan |= l[i] != l[i];
            best = max(best, key[i]);
        }
        nan = __any(nan);
        best = wave_max(best);
        const uint32_t top_bits = best & 0x80000000u ? best & 0x7FFFFFFFu : ~best;
        const float top = __builtin_bit_cast(float, top_bits);
        // exp(l - top): nothing where every expert is masked
        const bool none = top == -__builtin_inff();
        float all = 0.f, chosen = 0.f;
#pragma unroll
        for (int i = 0; i < MOE_MAX_EXPERTS / 64; i++) all += none ? 0.f : __expf(l[i] - top);
        all = wave_sum(all);
        float mine = 0.f;
        for (int j = 0; j < a.top_k; j++) {
            uint32_t high = 0;
#pragma unroll
            for (int i = 0; i < MOE_MAX_EXPERTS / 64; i++) high = max(high, key[i]);
            high = wave_max(high);
            int id = -1;
            float value = 0.f;
#pragma unroll
            for (int i = 0; i < MOE_MAX_EXPERTS / 64; i++) {
                const uint64_t who = __ballot(key[i] == high);
                if (id < 0 && who) {
                    const int at = __builtin_ctzll(who);
                    id = 64 * i + at;
                    value = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, l[i]), at));
                    if (lane == at) key[i] = 0;
                }
            }
            const float w = none ? 0.f : __expf(value - top);
            chosen += w;
            if (lane == j) {
                my_id[m] = id;
                mine = w;
            }
        }
        const float sum = a.renormalize ? chosen : all;
        my_weight[m] = nan ? __builtin_nanf("") : none ? 0.f : mine / sum;
        if (lane < a.top_k) {
            if (a.ids) a.ids[t * a.top_k + lane] = my_id[m];
            if (a.weights) a.weights[t * a.top_k + lane] = my_weight[m];
            // (a weight of 0 leaves the expert out, a NaN does not)
            if (my_weight[m] != 0.f) atomicOr(&s_tokens[my_id[m]], 1ull << t);
        }
    }
    __syncthreads();
    // experts in a row and their pairs: sums over the experts before, 64 at a time by the first wave
    if (wave == 0) {
        int experts = 0, pairs = 0;
        for (int i = 0; i < MOE_MAX_EXPERTS / 64; i++) {
            const uint64_t tokens = s_tokens[64 * i + lane];
            const int count = __builtin_popcountll(tokens);
            int before = count;  // inclusive sum over lanes
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(before, d, 64);
                if (lane >= d) before += o;
            }
            const uint64_t any = __ballot(count > 0);
            const int first = pairs + before - count;
            s_first[64 * i + lane] = first;
            if (count) {
                const int at = experts + __builtin_popcountll(any & ((1ull << lane) - 1));
                ws.plan->expert[at] = 64 * i + lane;
                ws.plan->first[at] = first;
                ws.plan->tokens[at] = tokens;
            }
            experts += __builtin_popcountll(any);
            pairs += __shfl(before, 63, 64);
        }
        if (lane == 0) ws.plan->experts = experts;
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MINE; m++) {
        const int t = wave + 16 * m;
        if (t < a.T && lane < a.top_k) {
            const int pair = my_weight[m] == 0.f ? -1 : s_first[my_id[m]] + __builtin_popcountll(s_tokens[my_id[m]] & ((1ull << t) - 1));
            ws.plan->pair[t * a.top_k + lane] = pair;
            ws.plan->weight[t * a.top_k + lane] = my_weight[m];
            if (pair >= 0) ws.plan->token[pair] = t;
        }
    }
}

// Sixteen weights as two operands of eight, in the activations' type.
template <class T> struct Operand;
template <> struct Operand<half_t> {
    typedef half8_t type;
    static __device__ __forceinline__ float4_t product(type w, type x, float4_t d) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, d, 0, 0, 0);
    }
};
template <> struct Operand<bf16_t> {
    typedef bf16x8_t type;
    static __device__ __forceinline__ float4_t product(type w, type x, float4_t d) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, d, 0, 0, 0);
    }
};
template <class T>
__device__ __forceinline__ void weights_of(i32x4_t v, typename Operand<T>::type &first, typename Operand<T>::type &second) {
#pragma unroll
    for (int d = 0; d < 4; d++)
#pragma unroll
        for (int b = 0; b < 4; b++) {
            const float one = (float)(int8_t)(v[d] >> (8 * b));
            if (d < 2) first[4 * d + b] = (T)one;
            else second[4 * (d - 2) + b] = (T)one;
        }
}

// The waves of a workgroup and the LDS that each has to itself; two workgroups on a CU.
constexpr int NW = 4, WAVE_LDS = 20 * 1024;

// Two blocks of 16 rows of 8-bit weights times up to 4 XC rows of activations: sum[block][16 rows], all of them in every
// lane's usual place.  The waves take 128 inputs in turn and add up at the end.  Each wave has a ring of stages in LDS,
// filled by copies past the registers: eight whole 128-byte pieces of weight rows a copy, four 256-byte pieces of activations.
// Unit c (16 bytes) of row r is at place c ^ (r / 2 % 8) of weights, c ^ r of activations: 16 rows one after the other have the
// same unit in different banks.
//   w_at[b], x_at(r): where a block's first row and activation row r begin in their buffers (row r >= rows: zeros).
template <class T, int XC, class At>
__device__ __forceinline__ void expert_sums(u32x4_t buffer_w, const uint32_t (&w_at)[2], u32x4_t buffer_x, At x_at, int rows, int n,
                                            char *s_ring, float4_t (&sum)[2][(XC + 3) / 4]) {
    typedef typename Operand<T>::type op_t;
    constexpr int NB = (XC + 3) / 4, STAGE = (4 + XC) * 1024, D = WAVE_LDS / STAGE;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    char *const ring = s_ring + wave * WAVE_LDS;
    uint32_t at_w[4], at_x[XC];
    int k_x[XC];  // the first input that the lane copies of activations
#pragma unroll
    for (int g = 0; g < 4; g++)
        at_w[g] = w_at[g >> 1] + (uint32_t)((g & 1) * 8 + (lane >> 3)) * (uint32_t)n + 16 * ((lane & 7) ^ ((g & 1) * 4 + (lane >> 4)));
#pragma unroll
    for (int g = 0; g < XC; g++) {
        const int r = 4 * g + (lane >> 4), unit = (lane & 15) ^ (r & 15);
        k_x[g] = r < rows ? 8 * unit : 1 << 30;
        at_x[g] = r < rows ? x_at(r) + 16 * unit : 0u;
    }
    const int stages = (n + 127) / 128, mine = (stages - wave + NW - 1) / NW;
    auto copy = [&](int s, int slot) {
        const uint32_t k = s * 128;
#pragma unroll
        for (int g = 0; g < 4; g++) copy_to_lds(buffer_w, at_w[g], k, ring + slot * STAGE + g * 1024);
        // (behind a row's end: zeros, whatever the weights have there)
#pragma unroll
        for (int g = 0; g < XC; g++)
            copy_to_lds(buffer_x, (int)k + k_x[g] >= n ? 0xFFFFFF00u : at_x[g], 2 * k, ring + slot * STAGE + (4 + g) * 1024);
    };
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
        for (int c = 0; c < NB; c++) sum[b][c] = float4_t{0.f, 0.f, 0.f, 0.f};
    const int row = lane & 15, hi = lane >> 4;
    auto products = [&](int slot, auto again) {
        const char *const stage = ring + slot * STAGE;
        i32x4_t w[2][2];
        op_t x[NB][4];
#pragma unroll
        for (int h = 0; h < 2; h++) {  // units hi and hi + 4: inputs 16 hi ... 16 hi + 15, and those 64 behind
#pragma unroll
            for (int b = 0; b < 2; b++)
                w[b][h] = *reinterpret_cast<const i32x4_t *>(stage + b * 2048 + row * 128 + (((4 * h + hi) ^ (row >> 1)) << 4));
#pragma unroll
            for (int c = 0; c < NB; c++)
#pragma unroll
                for (int o = 0; o < 2; o++)
                    x[c][2 * h + o] = *reinterpret_cast<const op_t *>(stage + 4096 + (XC < 4 ? row % (4 * XC) : 16 * c + row) * 256 +
                                                                     (((8 * h + 2 * hi + o) ^ (XC < 4 ? row % (4 * XC) : row)) << 4));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        again();
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int b = 0; b < 2; b++) {
                op_t first, second;
                weights_of<T>(w[b][h], first, second);
#pragma unroll
                for (int c = 0; c < NB; c++) {
                    sum[b][c] = Operand<T>::product(first, x[c][2 * h], sum[b][c]);
                    sum[b][c] = Operand<T>::product(second, x[c][2 * h + 1], sum[b][c]);
                }
            }
    };
#pragma unroll
    for (int d = 0; d < D; d++)
        if (d < mine) copy(wave + d * NW, d);
    int j = 0, slot = 0;
    for (; j + D < mine; j++) {
        __builtin_amdgcn_s_waitcnt(vmcnt_only((D - 1) * (4 + XC)));
        asm volatile("" ::: "memory");
        products(slot, [&] { copy(wave + (j + D) * NW, slot); });
        slot = slot + 1 == D ? 0 : slot + 1;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
    asm volatile("" ::: "memory");
    for (; j < mine; j++) {
        products(slot, [] {});
        slot = slot + 1 == D ? 0 : slot + 1;
    }
    __syncthreads();
    auto *const sums = reinterpret_cast<float4_t(*)[2 * NB][64]>(s_ring);
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
        for (int c = 0; c < NB; c++) sums[wave][b * NB + c][lane] = sum[b][c];
    __syncthreads();
    if (wave < NB) {  // a wave for 16 rows of activations
#pragma unroll
        for (int b = 0; b < 2; b++) {
            const int o = b * NB + wave;
            sum[b][0] = (sums[0][o][lane] + sums[1][o][lane]) + (sums[2][o][lane] + sums[3][o][lane]);
        }
    }
    __syncthreads();
}

// All rows of activations, 32 at a time: done(block sums, number of the row) in the lanes that have a row.
template <class T, class At, class Done>
__device__ __forceinline__ void expert_rows(u32x4_t buffer_w, const uint32_t (&w_at)[2], u32x4_t buffer_x, At x_at, int rows, int n,
                                            char *s_ring, Done done) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int r0 = 0; r0 < rows; r0 += 32) {
        auto some = [&](auto xc) {
            float4_t sum[2][(xc + 3) / 4];
            expert_sums<T, xc>(buffer_w, w_at, buffer_x, [&](int r) { return x_at(r0 + r); }, rows - r0, n, s_ring, sum);
            const int r = 16 * wave + (lane & 15);
            if (wave < (xc + 3) / 4) done(sum[0][0], sum[1][0], r0 + r, r < 4 * xc && r0 + r < rows);
        };
        if (rows - r0 <= 4) some(std::integral_constant<int, 1>{});
        else if (rows - r0 <= 8) some(std::integral_constant<int, 2>{});
        else if (rows - r0 <= 16) some(std::integral_constant<int, 4>{});
        else some(std::integral_constant<int, 8>{});
    }
}

// h of 16 rows of G and U of one expert.
template <class T> __global__ __launch_bounds__(NW * 64) void moe_up_kernel(MoeI8 a, Workspace ws) {
    __shared__ __attribute__((aligned(1024))) char s_ring[NW * WAVE_LDS];
    const Plan &plan = *ws.plan;
    const int u = blockIdx.y;
    if (u >= plan.experts) return;
    const int e = plan.expert[u], first = plan.first[u], count = __builtin_popcountll(plan.tokens[u]);
    const int i0 = blockIdx.x * 16, i = i0 + 4 * ((threadIdx.x & 63) >> 4);
    const u32x4_t buffer_w = buffer_of(a.W_up + (int64_t)e * 2 * a.f * a.n, (size_t)2 * a.f * a.n);
    const u32x4_t buffer_x = buffer_of(a.x, ((size_t)(a.T - 1) * a.ldx + a.n) * 2);
    const uint32_t w_at[2] = {(uint32_t)i0 * a.n, (uint32_t)(a.f + i0) * a.n};
    const float4_t sg = *reinterpret_cast<const float4_t *>(a.up_scale + (int64_t)e * 2 * a.f + i);
    const float4_t su = *reinterpret_cast<const float4_t *>(a.up_scale + (int64_t)e * 2 * a.f + a.f + i);
    expert_rows<T>(buffer_w, w_at, buffer_x, [&](int r) { return (uint32_t)plan.token[first + r] * (uint32_t)a.ldx * 2; }, count, a.n,
                   s_ring, [&](float4_t g, float4_t up, int r, bool there) {
        if (!there) return;
        bf16x4_t high, low;
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const float h = silu(g[c] * sg[c]) * (up[c] * su[c]);
            high[c] = (bf16_t)h;
            // (what is infinite or undefined has no rest)
            const float rest = h - (float)high[c];
            low[c] = (bf16_t)(__builtin_isfinite(rest) ? rest : 0.f);
        }
        bf16_t *to = ws.h + (int64_t)(first + r) * 2 * a.f + i;
        *reinterpret_cast<bf16x4_t *>(to) = high;
        *reinterpret_cast<bf16x4_t *>(to + a.f) = low;
    });
}

// D h of 32 rows of D of one expert.
__global__ __launch_bounds__(NW * 64) void moe_down_kernel(MoeI8 a, Workspace ws) {
    __shared__ __attribute__((aligned(1024))) char s_ring[NW * WAVE_LDS];
    const Plan &plan = *ws.plan;
    const int u = blockIdx.y;
    if (u >= plan.experts) return;
    const int e = plan.expert[u], first = plan.first[u], count = __builtin_popcountll(plan.tokens[u]);
    const int i0 = blockIdx.x * 32, i1 = min(i0 + 16, a.n - 16), i = i0 + 4 * ((threadIdx.x & 63) >> 4);  // (n may end with the first block)
    const u32x4_t buffer_w = buffer_of(a.W_down + (int64_t)e * a.n * a.f, (size_t)a.n * a.f);
    const u32x4_t buffer_x = buffer_of(ws.h + (int64_t)first * 2 * a.f, (size_t)count * 4 * a.f);
    const uint32_t w_at[2] = {(uint32_t)i0 * a.f, (uint32_t)i1 * a.f};
    const float4_t s0 = *reinterpret_cast<const float4_t *>(a.down_scale + (int64_t)e * a.n + i);
    const float4_t s1 = *reinterpret_cast<const float4_t *>(a.down_scale + (int64_t)e * a.n + i1 + (i - i0));
    expert_rows<bf16_t>(buffer_w, w_at, buffer_x, [&](int r) { return (uint32_t)r * (uint32_t)a.f * 2; }, 2 * count, a.f, s_ring,
                        [&](float4_t d0, float4_t d1, int r, bool there) {
        // (the two rows of one h are in neighbouring lanes)
#pragma unroll
        for (int c = 0; c < 4; c++) {
            const float one = d0[c], two = d1[c];
            d0[c] = one + __builtin_bit_cast(float, dpp<0xB1>(__builtin_bit_cast(uint32_t, one)));
            d1[c] = two + __builtin_bit_cast(float, dpp<0xB1>(__builtin_bit_cast(uint32_t, two)));
        }
        if (!there || (r & 1)) return;
        float *to = ws.parts + (int64_t)(first + r / 2) * a.n + i;
        *reinterpret_cast<float4_t *>(to) = d0 * s0;
        if (i0 + 16 < a.n) *reinterpret_cast<float4_t *>(to + 16) = d1 * s1;
    });
}

// y of a token: its experts' parts by descending weight.
template <class T> __global__ __launch_bounds__(256) void moe_join_kernel(MoeI8 a, Workspace ws) {
    const int t = blockIdx.y, i = 4 * (blockIdx.x * 256 + threadIdx.x);
    if (i >= a.n) return;
    float4_t y = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.top_k; j++) {
        const int pair = ws.plan->pair[t * a.top_k + j];
        if (pair >= 0) y += ws.plan->weight[t * a.top_k + j] * *reinterpret_cast<const float4_t *>(ws.parts + (int64_t)pair * a.n + i);
    }
    store_quad((T *)a.y + t * a.ldy, i, a.n, y);
}

template <class T> void launch_moe(const MoeI8 &a, const Workspace &ws, hipStream_t st) {
    hipLaunchKernelGGL((moe_logits_kernel<T>), dim3((a.E + 3) / 4, (a.T + 3) / 4), dim3(256), 0, st, a, ws.logits);
    hipLaunchKernelGGL(moe_choose_kernel, dim3(1), dim3(1024), 0, st, a, ws);
    const int experts = a.T * a.top_k < a.E ? a.T * a.top_k : a.E;
    hipLaunchKernelGGL((moe_up_kernel<T>), dim3(a.f / 16, experts), dim3(NW * 64), 0, st, a, ws);
    hipLaunchKernelGGL(moe_down_kernel, dim3((a.n + 31) / 32, experts), dim3(NW * 64), 0, st, a, ws);
    hipLaunchKernelGGL((moe_join_kernel<T>), dim3((a.n + 1023) / 1024, a.T), dim3(256), 0, st, a, ws);
}

}  // namespace

size_t moe_i8_workspace(int T, int n, int f, int E, int top_k) { return Workspace::bytes(T, n, f, E, top_k); }

hipError_t launch_moe_i8(const MoeI8 &a, void *ws, hipStream_t st) {
    if (a.type == TYPE_F16) launch_moe<half_t>(a, Workspace(ws, a), st);
    else launch_moe<bf16_t>(a, Workspace(ws, a), st);
    return hipGetLastError();
}

}  // namespace qtip

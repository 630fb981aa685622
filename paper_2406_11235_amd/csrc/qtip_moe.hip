// A mixture-of-experts layer for a few tokens.  For each token x:
//   l = R x + bias;  the top_k largest l, ties to the lowest expert;  p = softmax(l), over all experts or the chosen ones;
//   h_e = silu(G_e x) .* (U_e x);  y = sum over the chosen e of p_e D_e h_e
// with the experts' weights in 8 bits, a scale for each row, and activations in 16 bits.
//
// What bounds it is reading the chosen experts' weights, once each.  Four launches: logits; the choice; G, U and h; D and
// the sum.  The products run on the matrix cores with 16 rows of weights as one operand and 16 tokens as the other;
// weights become 16-bit floats on the way, exactly.  h lives in memory as the sum of two bf16 numbers (16 bits of mantissa at
// any size), so that y is what binary32 would give before its one rounding.
#include "qtip_device.h"
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
    float weight[MOE_MAX_TOKENS * MOE_MAX_TOP_K];  // by pair
    uint8_t token[MOE_MAX_TOKENS * MOE_MAX_TOP_K];
};

constexpr size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

struct Workspace {
    Plan *plan;
    float *logits;        // T x E
    bf16_t *h_high, *h_low;  // pairs x f
    static size_t bytes(int T, int f, int E, int top_k) {
        return round_up(sizeof(Plan)) + round_up((size_t)T * E * 4) + 2 * round_up((size_t)T * top_k * f * 2);
    }
    Workspace(void *at, const MoeI8 &a) {
        char *p = (char *)at;
        plan = (Plan *)p;
        p += round_up(sizeof(Plan));
        logits = (float *)p;
        p += round_up((size_t)a.T * a.E * 4);
        h_high = (bf16_t *)p;
        p += round_up((size_t)a.T * a.top_k * a.f * 2);
        h_low = (bf16_t *)p;
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
        if (t < a.T && lane < a.top_k && my_weight[m] != 0.f) {
            const int pair = s_first[my_id[m]] + __builtin_popcountll(s_tokens[my_id[m]] & ((1ull << t) - 1));
            ws.plan->weight[pair] = my_weight[m];
            ws.plan->token[pair] = (uint8_t)t;
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

// h of 16 rows of G and U of one expert: NW waves take 64 inputs in turn, for 16 tokens at a time.
template <class T, int NW> __global__ __launch_bounds__(NW * 64) void moe_up_kernel(MoeI8 a, Workspace ws) {
    typedef typename Operand<T>::type op_t;
    __shared__ float4_t s_sum[NW][2][64];
    const Plan &plan = *ws.plan;
    const int u = blockIdx.y;
    if (u >= plan.experts) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int e = plan.expert[u], first = plan.first[u], count = __builtin_popcountll(plan.tokens[u]);
    const int i0 = blockIdx.x * 16;
    const int8_t *g = a.W_up + ((int64_t)e * 2 * a.f + i0 + (lane & 15)) * a.n;
    const int8_t *up = g + (int64_t)a.f * a.n;
    for (int c0 = 0; c0 < count; c0 += 16) {
        const int pair = first + min(c0 + (lane & 15), count - 1);
        const T *x = (const T *)a.x + (int64_t)plan.token[pair] * a.ldx;
        float4_t sum[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        for (int c = wave * 64; c < a.n; c += NW * 64) {
            const int k = c + 16 * (lane >> 4);
            i32x4_t wg = {0, 0, 0, 0}, wu = {0, 0, 0, 0};
            op_t x0 = {}, x1 = {};
            if (k < a.n) {
                wg = *reinterpret_cast<const i32x4_t *>(g + k);
                wu = *reinterpret_cast<const i32x4_t *>(up + k);
                x0 = *reinterpret_cast<const op_t *>(x + k);
                x1 = *reinterpret_cast<const op_t *>(x + k + 8);
            }
            op_t w0, w1;
            weights_of<T>(wg, w0, w1);
            sum[0] = Operand<T>::product(w0, x0, sum[0]);
            sum[0] = Operand<T>::product(w1, x1, sum[0]);
            weights_of<T>(wu, w0, w1);
            sum[1] = Operand<T>::product(w0, x0, sum[1]);
            sum[1] = Operand<T>::product(w1, x1, sum[1]);
        }
        s_sum[wave][0][lane] = sum[0];
        s_sum[wave][1][lane] = sum[1];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int other = 1; other < NW; other++) {
                sum[0] += s_sum[other][0][lane];
                sum[1] += s_sum[other][1][lane];
            }
            if (c0 + (lane & 15) < count) {
                const int i = i0 + 4 * (lane >> 4);
                const float4_t sg = *reinterpret_cast<const float4_t *>(a.up_scale + (int64_t)e * 2 * a.f + i);
                const float4_t su = *reinterpret_cast<const float4_t *>(a.up_scale + (int64_t)e * 2 * a.f + a.f + i);
                bf16x4_t high, low;
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float h = silu(sum[0][r] * sg[r]) * (sum[1][r] * su[r]);
                    high[r] = (bf16_t)h;
                    // (what is infinite or undefined has no rest)
                    const float rest = h - (float)high[r];
                    low[r] = (bf16_t)(__builtin_isfinite(rest) ? rest : 0.f);
                }
                *reinterpret_cast<bf16x4_t *>(ws.h_high + (int64_t)pair * a.f + i) = high;
                *reinterpret_cast<bf16x4_t *>(ws.h_low + (int64_t)pair * a.f + i) = low;
            }
        }
        __syncthreads();
    }
}

// y of 16 outputs for all tokens, 16 at a time: the waves take 64 values of h of each chosen expert in turn.  A matrix
// operand's column is a token, zeros where it did not choose the expert.
template <class T, int NW> __global__ __launch_bounds__(NW * 64) void moe_down_kernel(MoeI8 a, Workspace ws) {
    __shared__ float4_t s_sum[NW][64];
    const Plan &plan = *ws.plan;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int i0 = blockIdx.x * 16, i = i0 + 4 * (lane >> 4);
    const int t = blockIdx.y * 16 + (lane & 15);
    const int experts = plan.experts;
    float4_t y = {0.f, 0.f, 0.f, 0.f};
    for (int u = 0; u < experts; u++) {
        const uint64_t tokens = plan.tokens[u];
        if (((tokens >> (blockIdx.y * 16)) & 0xFFFF) == 0) continue;
        const int e = plan.expert[u];
        const bool mine = (tokens >> t) & 1;
        const int pair = plan.first[u] + __builtin_popcountll(tokens & ((1ull << t) - 1));
        const int8_t *w = a.W_down + ((int64_t)e * a.n + i0 + (lane & 15)) * a.f;
        const bf16_t *high = ws.h_high + (int64_t)(mine ? pair : 0) * a.f, *low = ws.h_low + (int64_t)(mine ? pair : 0) * a.f;
        float4_t sum = {0.f, 0.f, 0.f, 0.f};
        for (int c = wave * 64; c < a.f; c += NW * 64) {
            const int k = c + 16 * (lane >> 4);
            i32x4_t v = {0, 0, 0, 0};
            bf16x8_t h0 = {}, h1 = {}, l0 = {}, l1 = {};
            if (k < a.f) {
                v = *reinterpret_cast<const i32x4_t *>(w + k);
                if (mine) {
                    h0 = *reinterpret_cast<const bf16x8_t *>(high + k);
                    h1 = *reinterpret_cast<const bf16x8_t *>(high + k + 8);
                    l0 = *reinterpret_cast<const bf16x8_t *>(low + k);
                    l1 = *reinterpret_cast<const bf16x8_t *>(low + k + 8);
                }
            }
            bf16x8_t w0, w1;
            weights_of<bf16_t>(v, w0, w1);
            sum = Operand<bf16_t>::product(w0, l0, sum);
            sum = Operand<bf16_t>::product(w1, l1, sum);
            sum = Operand<bf16_t>::product(w0, h0, sum);
            sum = Operand<bf16_t>::product(w1, h1, sum);
        }
        if (mine) {
            const float4_t scale = *reinterpret_cast<const float4_t *>(a.down_scale + (int64_t)e * a.n + i);
            y += sum * (scale * plan.weight[pair]);
        }
    }
    s_sum[wave][lane] = y;
    __syncthreads();
    if (wave != 0 || t >= a.T) return;
#pragma unroll
    for (int other = 1; other < NW; other++) y += s_sum[other][lane];
    store_quad((T *)a.y + t * a.ldy, i, a.n, y);
}

template <class T> void launch_moe(const MoeI8 &a, const Workspace &ws, hipStream_t st) {
    hipLaunchKernelGGL((moe_logits_kernel<T>), dim3((a.E + 3) / 4, (a.T + 3) / 4), dim3(256), 0, st, a, ws.logits);
    hipLaunchKernelGGL(moe_choose_kernel, dim3(1), dim3(1024), 0, st, a, ws);
    const int experts = a.T * a.top_k < a.E ? a.T * a.top_k : a.E;
    hipLaunchKernelGGL((moe_up_kernel<T, 4>), dim3(a.f / 16, experts), dim3(256), 0, st, a, ws);
    hipLaunchKernelGGL((moe_down_kernel<T, 16>), dim3(a.n / 16, (a.T + 15) / 16), dim3(1024), 0, st, a, ws);
}

}  // namespace

size_t moe_i8_workspace(int T, int f, int E, int top_k) { return Workspace::bytes(T, f, E, top_k); }

hipError_t launch_moe_i8(const MoeI8 &a, void *ws, hipStream_t st) {
    if (a.type == TYPE_F16) launch_moe<half_t>(a, Workspace(ws, a), st);
    else launch_moe<bf16_t>(a, Workspace(ws, a), st);
    return hipGetLastError();
}

}  // namespace qtip

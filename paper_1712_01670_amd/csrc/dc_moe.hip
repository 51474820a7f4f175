// A mixture-of-experts layer for a few tokens (a row per video stream): a router chooses top_k of the experts for every token,
// an expert is a pair of fully-connected layers, and the token's output is the sum of its experts', weighted by the router's
// softmax.  What bounds it is the weights of the chosen experts, each of which is read once for up to 64 tokens; three launches:
// the choice, the experts' first layers, their second layers with the weighted sum.
#include <hip/hip_bf16.h>

#include <algorithm>

#include "dc_internal.h"

namespace dc {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

struct Moe {
    const void* x;                     // [n_tokens][cin]
    const void* router;                // [experts][cin]
    const float* router_bias;
    const void* up;                    // [experts][halves][hidden][cin]
    const float *up_scale, *up_bias;   // [experts][halves][hidden]
    const void* down;                  // [experts][cout][hidden]
    const float *down_scale, *down_bias;   // [experts][cout]
    void* out;                         // [n_tokens][cout]
    int32_t* choice;                   // [n_tokens][top_k]: an expert, or -1
    float* gate;                       // [n_tokens][top_k]
    unsigned char* hidden_out;         // [n_tokens * top_k]: the experts' hidden values (hidden_row)
    int n_tokens, experts, top_k, cin, hidden, cout, renormalize;
    int hidden_pad;                    // hidden rounded up to 16, zeros behind it
};

constexpr int kMoeTokens = 64;         // tokens that share one pass over the weights
constexpr int kMoeWaves = 8;

// PE elements (16 bytes of the weights) from k0 on, zeros behind the row's end.  Any address the type allows.
template <typename E, int N>
struct Piece { E v[N]; };
template <int N, typename E>
__device__ __forceinline__ Piece<E, N> piece(const E* __restrict__ row, int k0, int K) {
    Piece<E, N> p;
    if (k0 + N <= K) {
        __builtin_memcpy(&p, row + k0, sizeof p);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) p.v[e] = k0 + e < K ? row[k0 + e] : E{};
    }
    return p;
}

// acc[channel][token] += sum over a piece; fp32 tokens: one product of four k a step; bf16: eight a lane.
template <int N>
__device__ __forceinline__ void mma(const Piece<float, N>& w, const Piece<float, N>& x, floatx4& acc) {
#pragma unroll
    for (int e = 0; e < N; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[e], x.v[e], acc, 0, 0, 0);
}
template <int N>
__device__ __forceinline__ void mma(const Piece<uint16_t, N>& w, const Piece<uint16_t, N>& x, floatx4& acc) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
        bf16x8 a, b;
        __builtin_memcpy(&a, &w.v[8 * i], 16);
        __builtin_memcpy(&b, &x.v[8 * i], 16);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
    }
}
// Weights as operands of the tokens' type; 8-bit integers are exact in either.
template <int N>
__device__ __forceinline__ Piece<float, N> operand(const Piece<float, N>& w, float) { return w; }
template <int N>
__device__ __forceinline__ Piece<uint16_t, N> operand(const Piece<uint16_t, N>& w, uint16_t) { return w; }
template <int N>
__device__ __forceinline__ Piece<float, N> operand(const Piece<int8_t, N>& w, float) {
    Piece<float, N> p;
#pragma unroll
    for (int e = 0; e < N; ++e) p.v[e] = (float)w.v[e];
    return p;
}
template <int N>
__device__ __forceinline__ Piece<uint16_t, N> operand(const Piece<int8_t, N>& w, uint16_t) {
    Piece<uint16_t, N> p;
#pragma unroll
    for (int e = 0; e < N; ++e) p.v[e] = (uint16_t)(__float_as_uint((float)w.v[e]) >> 16);
    return p;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, __float2bfloat16(v)); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(uint16_t* p, float v) { *p = to_bf16(v); }

// ---- the choice ---------------------------------------------------------------------------------------------------------
// Order of the logits as whole numbers: a NaN stands below every number, -inf is 0 and never chosen.
__device__ __forceinline__ uint32_t logit_key(float l) {
    if (l != l) return 1;
    const uint32_t u = __float_as_uint(l + 0.f);     // -0 is 0
    if (u == 0xff800000u) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A workgroup takes a token: its wavefronts deal the experts among themselves, the first one chooses.
template <typename T>
__global__ __launch_bounds__(256) void moe_choose_kernel(Moe P) {
    __shared__ float logits[kMoeMaxExperts];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, token = blockIdx.x;
    const T* const x = static_cast<const T*>(P.x) + (size_t)token * P.cin;
    for (int e = wave; e < P.experts; e += 4) {
        const T* const w = static_cast<const T*>(P.router) + (size_t)e * P.cin;
        float sum = 0.f;
        for (int k = lane; k < P.cin; k += 64) sum = fmaf(to_float(x[k]), to_float(w[k]), sum);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) logits[e] = sum + (P.router_bias ? P.router_bias[e] : 0.f);
    }
    __syncthreads();
    if (wave != 0) return;
    constexpr int N = kMoeMaxExperts / 64;
    float top = -INFINITY, sum = 0.f;
    uint32_t key[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * 64 + lane;
        key[i] = e < P.experts ? logit_key(logits[e]) : 0;
        if (e < P.experts) top = fmaxf(top, logits[e]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * 64 + lane;
        if (e < P.experts && logits[e] != -INFINITY) sum += expf(logits[e] - top);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
    float mine = 0.f, chosen = 0.f;                  // lane j keeps choice j
    int expert = -1;
    for (int j = 0; j < P.top_k; ++j) {
        unsigned long long best = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const unsigned long long c = (unsigned long long)key[i] << 32 | (uint32_t)~(i * 64 + lane);      // equal: the lowest index
            if (key[i] && c > best) best = c;
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            const unsigned long long o = __shfl_xor(best, d);
            best = o > best ? o : best;
        }
        if (best == 0) break;
        const int e = (int)~(uint32_t)best;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * 64 + lane == e) key[i] = 0;
        const float g = expf(logits[e] - top) / sum;
        chosen += g;
        if (lane == j) { mine = g; expert = e; }
    }
    if (lane < P.top_k) {
        P.choice[(size_t)token * P.top_k + lane] = expert;
        P.gate[(size_t)token * P.top_k + lane] = expert >= 0 && P.renormalize ? mine / chosen : mine;
    }
}

// ---- the experts ----------------------------------------------------------------------------------------------------------
// The slots (token * top_k + choice) of a group of kMoeTokens tokens, by expert: which experts have any, and their slots in
// order.  Made by every workgroup for itself.
struct Chosen {
    uint32_t has[kMoeMaxExperts / 32];
    int slot[kMoeTokens];              // of one expert
    int n;
};
__device__ __forceinline__ void find_experts(const Moe& P, Chosen& C, int t0, int n_tok) {
    for (int i = threadIdx.x; i < kMoeMaxExperts / 32; i += blockDim.x) C.has[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n_tok * P.top_k; i += blockDim.x) {
        const int e = P.choice[(size_t)t0 * P.top_k + i];
        if (e >= 0) atomicOr(&C.has[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
}
// The a-th expert that has tokens, or -1.
__device__ __forceinline__ int nth_expert(const Chosen& C, int a) {
    for (int i = 0; i < kMoeMaxExperts / 32; ++i) {
        uint32_t m = C.has[i];
        const int c = __popc(m);
        if (a >= c) { a -= c; continue; }
        for (; a > 0; --a) m &= m - 1;
        return i * 32 + __ffs((int)m) - 1;
    }
    return -1;
}
// Slots of expert e, by the first wavefront: a lane per token.
__device__ __forceinline__ void list_slots(const Moe& P, Chosen& C, int e, int t0, int n_tok) {
    if (threadIdx.x < 64) {
        int at = -1;
        if ((int)threadIdx.x < n_tok)
            for (int j = 0; j < P.top_k; ++j)
                if (P.choice[(size_t)(t0 + threadIdx.x) * P.top_k + j] == e) at = (t0 + threadIdx.x) * P.top_k + j;
        const unsigned long long m = __ballot(at >= 0);
        if (at >= 0) C.slot[__popcll(m & ((1ull << threadIdx.x) - 1))] = at;
        if (threadIdx.x == 0) C.n = __popcll(m);
    }
    __syncthreads();
}

// Hidden values of a slot: fp32, or two bf16 numbers each (the value's rounding and what that leaves) in two rows, so that the
// second product sees 16 bits of them: the layer's output is rounded once, as if they were fp32.
template <typename T>
__device__ __forceinline__ T* hidden_row(const Moe& P, int slot) {
    return reinterpret_cast<T*>(P.hidden_out) + (size_t)slot * P.hidden_pad * (sizeof(T) == 2 ? 2 : 1);
}

// 16 channels of an expert's first layer for all its tokens of the group; K is dealt among the wavefronts.
template <typename T, typename W, int NB, bool GATED>
__global__ __launch_bounds__(kMoeWaves * 64) void moe_up_kernel(Moe P) {
    constexpr int PE = 16 / sizeof(W), HALVES = GATED ? 2 : 1;
    __shared__ Chosen C;
    __shared__ floatx4 red[kMoeWaves][NB][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16, t0 = blockIdx.z * kMoeTokens, n_tok = min(kMoeTokens, P.n_tokens - t0);
    find_experts(P, C, t0, n_tok);
    const int e = nth_expert(C, blockIdx.y);
    if (e < 0) return;
    list_slots(P, C, e, t0, n_tok);
    const int n = C.n, n_blocks = (n + 15) / 16;
    const W* wrow[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h)       // channels past the end repeat the last one (their values are set to zero)
        wrow[h] = static_cast<const W*>(P.up) + (((size_t)e * HALVES + h) * P.hidden + min(o0 + l16, P.hidden - 1)) * P.cin;
    const T* xrow[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) xrow[j] = static_cast<const T*>(P.x) + (size_t)(C.slot[min(j * 16 + l16, n - 1)] / P.top_k) * P.cin;
    floatx4 acc[HALVES][NB];
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[h][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int k = wave * 4 * PE; k < P.cin; k += kMoeWaves * 4 * PE) {
        Piece<W, PE> w[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) w[h] = piece<PE>(wrow[h], k + g * PE, P.cin);
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (j < n_blocks) {
                const Piece<T, PE> x = piece<PE>(xrow[j], k + g * PE, P.cin);
#pragma unroll
                for (int h = 0; h < HALVES; ++h) mma(operand(w[h], T{}), x, acc[h][j]);
            }
    }
    floatx4 sum[HALVES][(NB + kMoeWaves - 1) / kMoeWaves];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        if (h) __syncthreads();
#pragma unroll
        for (int j = 0; j < NB; ++j) red[wave][j][lane] = acc[h][j];
        __syncthreads();
        if (wave < NB) {
            sum[h][0] = red[0][wave][lane];
#pragma unroll
            for (int v = 1; v < kMoeWaves; ++v) sum[h][0] += red[v][wave][lane];
        }
    }
    const int at = wave * 16 + l16;        // wavefront j: block j of the tokens
    if (wave >= NB || at >= n) return;
    const int slot = C.slot[at];
    T* const out = hidden_row<T>(P, slot) + o0 + g * 4;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int o = o0 + g * 4 + r;
        float v = 0.f;
        if (o < P.hidden) {
            float u[HALVES];
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const size_t c = ((size_t)e * HALVES + h) * P.hidden + o;
                u[h] = sum[h][0][r] * (sizeof(W) == 1 ? P.up_scale[c] : 1.f) + (P.up_bias ? P.up_bias[c] : 0.f);
            }
            if constexpr (GATED) v = u[0] / (1.f + expf(-u[0])) * u[HALVES - 1];
            else v = u[0] > 0.f || u[0] != u[0] ? u[0] : 0.f;
        }
        store(out + r, v);
        if constexpr (sizeof(T) == 2) {
            const float high = to_float(to_bf16(v));
            store(out + P.hidden_pad + r, fabsf(high) < INFINITY || high != high ? v - high : 0.f);
        }
    }
}

// 16 channels of the outputs of a group of tokens: the experts one after another, their contributions added per token in LDS
// (a copy per wavefront, which has its share of K), in the order of the experts.
template <typename T, typename W, int NB>
__global__ __launch_bounds__(kMoeWaves * 64) void moe_down_kernel(Moe P) {
    constexpr int PE = 16 / sizeof(W);
    __shared__ Chosen C;
    __shared__ float y[kMoeWaves][NB * 16][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16, t0 = blockIdx.z * kMoeTokens, n_tok = min(kMoeTokens, P.n_tokens - t0);
    for (int i = tid; i < kMoeWaves * NB * 256; i += kMoeWaves * 64) (&y[0][0][0])[i] = 0.f;
    find_experts(P, C, t0, n_tok);
    for (int a = 0;; ++a) {
        const int e = nth_expert(C, a);
        if (e < 0) break;
        list_slots(P, C, e, t0, n_tok);
        const int n = C.n, n_blocks = (n + 15) / 16;
        const W* const wrow = static_cast<const W*>(P.down) + ((size_t)e * P.cout + min(o0 + l16, P.cout - 1)) * P.hidden;
        const T* hrow[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) hrow[j] = hidden_row<T>(P, C.slot[min(j * 16 + l16, n - 1)]);
        floatx4 acc[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int k = wave * 4 * PE; k < P.hidden; k += kMoeWaves * 4 * PE) {
            const Piece<T, PE> w = operand(piece<PE>(wrow, k + g * PE, P.hidden), T{});
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (j < n_blocks) {
                    mma(w, piece<PE>(hrow[j], k + g * PE, P.hidden_pad), acc[j]);
                    if constexpr (sizeof(T) == 2) mma(w, piece<PE>(hrow[j] + P.hidden_pad, k + g * PE, P.hidden_pad), acc[j]);
                }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int at = j * 16 + l16;
            if (at >= n) continue;
            const int slot = C.slot[at], token = slot / P.top_k - t0;
            const float gate = P.gate[slot];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int o = min(o0 + g * 4 + r, P.cout - 1);
                float v = acc[j][r] * (sizeof(W) == 1 ? P.down_scale[(size_t)e * P.cout + o] : 1.f);
                if (wave == 0 && P.down_bias) v += P.down_bias[(size_t)e * P.cout + o];
                y[wave][token][g * 4 + r] += gate * v;
            }
        }
        __syncthreads();
    }
    __syncthreads();
    for (int i = tid; i < n_tok * 16; i += kMoeWaves * 64) {
        const int token = i >> 4, o = o0 + (i & 15);
        if (o >= P.cout) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kMoeWaves; ++w) v += y[w][token][i & 15];
        store(static_cast<T*>(P.out) + (size_t)(t0 + token) * P.cout + o, v);
    }
}

template <typename T, typename W, int NB>
hipError_t moe_experts(const Moe& P, bool gated, hipStream_t st) {
    const unsigned groups = (unsigned)((P.n_tokens + kMoeTokens - 1) / kMoeTokens);
    const unsigned active = (unsigned)std::min(P.experts, std::min(P.n_tokens, kMoeTokens) * P.top_k);      // at most
    const dim3 up((unsigned)((P.hidden + 15) / 16), active, groups), down((unsigned)((P.cout + 15) / 16), 1, groups), block(kMoeWaves * 64);
    if (gated) hipLaunchKernelGGL((moe_up_kernel<T, W, NB, true>), up, block, 0, st, P);
    else hipLaunchKernelGGL((moe_up_kernel<T, W, NB, false>), up, block, 0, st, P);
    hipLaunchKernelGGL((moe_down_kernel<T, W, NB>), down, block, 0, st, P);
    return hipGetLastError();
}

template <typename T, typename W>
hipError_t moe_run(const Moe& P, bool gated, hipStream_t st) {
    hipLaunchKernelGGL((moe_choose_kernel<T>), dim3((unsigned)P.n_tokens), dim3(256), 0, st, P);
    const int most = std::min(P.n_tokens, kMoeTokens);
    if (most <= 16) return moe_experts<T, W, 1>(P, gated, st);
    if (most <= 32) return moe_experts<T, W, 2>(P, gated, st);
    return moe_experts<T, W, 4>(P, gated, st);
}

}  // namespace

size_t moe_workspace(const dc_moe& m, int n_tokens) {
    const size_t slots = (size_t)n_tokens * m.top_k;
    return 2 * align_up(slots * 4, 256) + align_up(slots * ((m.hidden + 15) / 16 * 16) * 4, 256);
}

hipError_t launch_moe(const dc_moe& m, const dc_moe_weights& w, const void* in, void* out, int32_t* experts, float* gates, int n_tokens, int dtype,
                      void* ws, hipStream_t st) {
    Moe P;
    const size_t slots = (size_t)n_tokens * m.top_k;
    unsigned char* const base = static_cast<unsigned char*>(ws);
    P.x = in; P.router = w.router; P.router_bias = w.router_bias;
    P.up = w.up; P.up_scale = w.up_scale; P.up_bias = w.up_bias;
    P.down = w.down; P.down_scale = w.down_scale; P.down_bias = w.down_bias;
    P.out = out;
    P.choice = experts ? experts : reinterpret_cast<int32_t*>(base);
    P.gate = gates ? gates : reinterpret_cast<float*>(base + align_up(slots * 4, 256));
    P.hidden_out = base + 2 * align_up(slots * 4, 256);
    P.n_tokens = n_tokens; P.experts = m.experts; P.top_k = m.top_k; P.cin = m.cin; P.hidden = m.hidden; P.cout = m.cout;
    P.renormalize = m.renormalize; P.hidden_pad = (m.hidden + 15) / 16 * 16;
    const bool gated = m.act == DC_MOE_GATED;
    if (dtype == DC_BF16) return m.wtype == DC_I8 ? moe_run<uint16_t, int8_t>(P, gated, st) : moe_run<uint16_t, uint16_t>(P, gated, st);
    return m.wtype == DC_I8 ? moe_run<float, int8_t>(P, gated, st) : moe_run<float, float>(P, gated, st);
}

}  // namespace dc

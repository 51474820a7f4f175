// A mixture-of-experts layer for a few tokens (a row per video stream): a router chooses top_k of the experts for every token,
// an expert is a pair of fully-connected layers, and the token's output is the sum of its experts', weighted by the router's
// softmax.  What bounds it is the weights of the chosen experts, each of which is read once for up to 64 tokens; four launches:
// the choice, the experts' first layers, their second layers, the weighted sum.
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
    int hidden_pad, cout_pad;          // hidden rounded up to 16, zeros behind it; cout rounded up to 4
    float* slot_out;                   // [n_tokens * top_k][cout_pad]: the experts' outputs
};

constexpr int kMoeTokens = 64;         // tokens that share one pass over the weights
constexpr int kMoeWaves = 8;

// N elements of a row from k0 on, at any address the type allows; zeros behind the row's end.
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

// A wavefront's operand for 4 * PE values of K, PE of them a lane (16 bytes of weights): one or more fragments of the matrix
// instruction, which takes 8 bf16 or 1 fp32 of a lane.  8-bit integers are exact in either.
template <typename T, typename W>
struct Operand {
    static constexpr int PE = 16 / sizeof(W), V = PE * sizeof(T) / 16;     // V: 16-byte vectors
    uintx4 v[V];
    // of the tokens' own type
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, p, sizeof v); }
    __device__ __forceinline__ void load(const T* row, int k0, int K) {
        const Piece<T, PE> t = piece<PE>(row, k0, K);
        __builtin_memcpy(v, &t, sizeof v);
    }
    // from weights as they lie in memory
    __device__ __forceinline__ explicit Operand(const uintx4& w) {
        if constexpr (sizeof(T) == sizeof(W)) {
            v[0] = w;
        } else {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = __float_as_uint((float)(int8_t)(w[d] >> (8 * e)));
                if constexpr (sizeof(T) == 4) v[d] = uintx4{f[0], f[1], f[2], f[3]};
                else {
                    v[d / 2][d % 2 * 2] = __builtin_amdgcn_perm(f[1], f[0], 0x07060302u);          // the upper halves are the bf16 numbers
                    v[d / 2][d % 2 * 2 + 1] = __builtin_amdgcn_perm(f[3], f[2], 0x07060302u);
                }
            }
        }
    }
    __device__ __forceinline__ Operand() {}
};
// acc[channel][token] += the sum over the operands' K
template <typename T, typename W>
__device__ __forceinline__ void mma(const Operand<T, W>& w, const Operand<T, W>& x, floatx4& acc) {
#pragma unroll
    for (int i = 0; i < Operand<T, W>::V; ++i) {
        if constexpr (sizeof(T) == 2) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.v[i]), __builtin_bit_cast(bf16x8, x.v[i]), acc, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.v[i][e]), __uint_as_float(x.v[i][e]), acc, 0, 0, 0);
        }
    }
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

// A workgroup takes a token: its wavefronts deal the experts among themselves, four at a time, the first one chooses.
constexpr int kRouterWaves = 8;
template <typename T>
__global__ __launch_bounds__(kRouterWaves * 64) void moe_choose_kernel(Moe P) {
    constexpr int VE = 16 / sizeof(T), EB = 4;
    __shared__ float logits[kMoeMaxExperts];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, token = blockIdx.x;
    const T* const x = static_cast<const T*>(P.x) + (size_t)token * P.cin;
    const T* const router = static_cast<const T*>(P.router);
    for (int e0 = wave * EB; e0 < P.experts; e0 += kRouterWaves * EB) {
        float sum[EB] = {};
        const T* w[EB];
#pragma unroll
        for (int i = 0; i < EB; ++i) w[i] = router + (size_t)min(e0 + i, P.experts - 1) * P.cin;
#pragma unroll 2
        for (int k = lane * VE; k < P.cin; k += 64 * VE) {
            const Piece<T, VE> xv = piece<VE>(x, k, P.cin);
#pragma unroll
            for (int i = 0; i < EB; ++i) {
                const Piece<T, VE> wv = piece<VE>(w[i], k, P.cin);
#pragma unroll
                for (int e = 0; e < VE; ++e) sum[i] = fmaf(to_float(xv.v[e]), to_float(wv.v[e]), sum[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < EB; ++i) {
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) sum[i] += __shfl_xor(sum[i], d);
            if (lane == i && e0 + i < P.experts) logits[e0 + i] = sum[i] + (P.router_bias ? P.router_bias[e0 + i] : 0.f);
        }
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

// The product of 32 channels of an expert (gated: of 16 in either half) with all its tokens of a group: relu or gate of the first
// layer into the hidden values, or the second layer into the slots' outputs.  The weights are what has to come from memory, once:
// they go straight into operands (16 rows of 64 bytes an instruction), three pieces of a wavefront ahead, and K is dealt among the
// wavefronts by pairs of pieces, whole cache lines; their sums are added through LDS in a fixed order.  The tokens' rows come from
// L2, a piece ahead, once for both tiles of weights.
enum { kUpRelu = 0, kUpGated = 1, kDown = 2 };
template <typename T, typename W, int KIND, int MOST>
__global__ __launch_bounds__(kMoeWaves * 64) void moe_expert_kernel(Moe P) {
    typedef Operand<T, W> Op;
    constexpr int PE = Op::PE, HALVES = KIND == kUpGated ? 2 : 1, R = 2, CT = R / HALVES;
    constexpr bool DOWN = KIND == kDown, TWO = DOWN && sizeof(T) == 2;      // TWO: a row is two
    __shared__ Chosen C;
    __shared__ floatx4 red[kMoeWaves][R][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int channels = DOWN ? P.cout : P.hidden, K = DOWN ? P.hidden : P.cin, row_end = DOWN ? P.hidden_pad : P.cin;
    const int o0 = blockIdx.x * (CT * 16), t0 = blockIdx.z * kMoeTokens, n_tok = min(kMoeTokens, P.n_tokens - t0);
    find_experts(P, C, t0, n_tok);
    const int e = nth_expert(C, blockIdx.y);
    if (e < 0) return;
    list_slots(P, C, e, t0, n_tok);
    const int n = C.n, pieces = (K + 4 * PE - 1) / (4 * PE), whole = K / (4 * PE);
    const W* wrow[R];                      // tile r: half r / CT, channels 16 (r % CT) on; past the end the last channel again
#pragma unroll
    for (int r = 0; r < R; ++r)
        wrow[r] = static_cast<const W*>(DOWN ? P.down : P.up) + (((size_t)e * HALVES + r / CT) * channels + min(o0 + r % CT * 16 + l16, channels - 1)) * K + g * PE;
    auto product = [&](auto blocks) {
        constexpr int NB = decltype(blocks)::value;
        const T* xrow[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int slot = C.slot[min(j * 16 + l16, n - 1)];
            xrow[j] = (DOWN ? hidden_row<T>(P, slot) : static_cast<const T*>(P.x) + (size_t)(slot / P.top_k) * P.cin) + g * PE;
        }
        // piece i of this wavefront
        auto at = [&](int i) { return (wave + i / 2 * kMoeWaves) * 2 + i % 2; };
        uintx4 w[4][R];
        Op x[2][NB], low[2][TWO ? NB : 1];
        auto fetch_w = [&](uintx4 (&to)[R], int p) {
            if (p < whole) {
#pragma unroll
                for (int r = 0; r < R; ++r) __builtin_memcpy(&to[r], wrow[r] + p * (4 * PE), 16);
            } else if (p < pieces) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const Piece<W, PE> t = piece<PE>(wrow[r], p * (4 * PE), K - g * PE);
                    __builtin_memcpy(&to[r], &t, 16);
                }
            }
        };
        auto fetch_x = [&](int b, int p) {
            if (p < whole) {
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    x[b][j].load(xrow[j] + p * (4 * PE));
                    if constexpr (TWO) low[b][j].load(xrow[j] + P.hidden_pad + p * (4 * PE));
                }
            } else if (p < pieces) {
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    x[b][j].load(xrow[j], p * (4 * PE), row_end - g * PE);
                    if constexpr (TWO) low[b][j].load(xrow[j] + P.hidden_pad, p * (4 * PE), row_end - g * PE);
                }
            }
        };
        floatx4 acc[R][NB];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[r][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        fetch_w(w[0], at(0));
        fetch_w(w[1], at(1));
        fetch_x(0, at(0));
        fetch_w(w[2], at(2));
        for (int i = 0; at(i) < pieces; i += 4) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                fetch_x((d + 1) & 1, at(i + d + 1));           // (loads come back in order: the rows before the weights further ahead)
                fetch_w(w[(d + 3) & 3], at(i + d + 3));
                __builtin_amdgcn_sched_barrier(0);
                if (at(i + d) < pieces) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const Op o(w[d][r]);
#pragma unroll
                        for (int j = 0; j < NB; ++j) {
                            mma(o, x[d & 1][j], acc[r][j]);
                            if constexpr (TWO) mma(o, low[d & 1][j], acc[r][j]);
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (j) __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) red[wave][r][lane] = acc[r][j];
            __syncthreads();
            const int at = j * 16 + l16, ct = wave;            // wavefront ct: tile ct of the channels
            if (ct >= CT || at >= n) continue;
            const int slot = C.slot[at], c0 = o0 + ct * 16 + g * 4;
            floatx4 sum[HALVES];
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                sum[h] = red[0][h * CT + ct][lane];
#pragma unroll
                for (int v = 1; v < kMoeWaves; ++v) sum[h] += red[v][h * CT + ct][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const size_t c = ((size_t)e * HALVES + h) * channels + min(c0 + i, channels - 1);
                    const float* const bias = DOWN ? P.down_bias : P.up_bias;
                    sum[h][i] = sum[h][i] * (sizeof(W) == 1 ? (DOWN ? P.down_scale : P.up_scale)[c] : 1.f) + (bias ? bias[c] : 0.f);
                }
            }
            if constexpr (DOWN) {
                if (c0 < P.cout_pad) *reinterpret_cast<floatx4*>(P.slot_out + (size_t)slot * P.cout_pad + c0) = sum[0];
            } else {
                T* const out = hidden_row<T>(P, slot) + c0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = sum[0][i];
                    float v;
                    if constexpr (KIND == kUpGated) v = u / (1.f + expf(-u)) * sum[HALVES - 1][i];
                    else v = u > 0.f || u != u ? u : 0.f;
                    if (c0 + i >= P.hidden) v = 0.f;
                    if (c0 + i >= P.hidden_pad) continue;
                    store(out + i, v);
                    if constexpr (sizeof(T) == 2) {
                        const float high = to_float(to_bf16(v));
                        store(out + P.hidden_pad + i, fabsf(high) < INFINITY || high != high ? v - high : 0.f);
                    }
                }
            }
        }
    };
    if (MOST == 1 || n <= 16) product(std::integral_constant<int, 1>());
    else if (n <= 32) product(std::integral_constant<int, 2>());
    else product(std::integral_constant<int, 4>());
}

// out[token] = sum over its choices of gate * the slot's output
template <typename T>
__global__ __launch_bounds__(256) void moe_combine_kernel(Moe P) {
    const int c = (blockIdx.x * 256 + threadIdx.x) * 4, token = blockIdx.y;
    if (c >= P.cout) return;
    floatx4 sum{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < P.top_k; ++j) {
        const size_t slot = (size_t)token * P.top_k + j;
        if (P.choice[slot] < 0) break;                         // (the places behind it are empty too)
        const floatx4 y = *reinterpret_cast<const floatx4*>(P.slot_out + slot * P.cout_pad + c);
        const float gate = P.gate[slot];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = fmaf(gate, y[i], sum[i]);
    }
    T* const out = static_cast<T*>(P.out) + (size_t)token * P.cout + c;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < P.cout) store(out + i, sum[i]);
}

template <typename T, typename W, int KIND>
hipError_t expert_launch(const Moe& P, hipStream_t st) {
    const unsigned groups = (unsigned)((P.n_tokens + kMoeTokens - 1) / kMoeTokens);
    const unsigned active = (unsigned)std::min(P.experts, std::min(P.n_tokens, kMoeTokens) * P.top_k);      // at most
    const unsigned tiles = (unsigned)((KIND == kDown ? P.cout : P.hidden) + (KIND == kUpGated ? 15 : 31)) / (KIND == kUpGated ? 16 : 32);
    const dim3 grid(tiles, active, groups), block(kMoeWaves * 64);
    if (P.n_tokens <= 16) hipLaunchKernelGGL((moe_expert_kernel<T, W, KIND, 1>), grid, block, 0, st, P);
    else hipLaunchKernelGGL((moe_expert_kernel<T, W, KIND, 4>), grid, block, 0, st, P);
    return hipGetLastError();
}

template <typename T, typename W>
hipError_t moe_run(const Moe& P, bool gated, hipStream_t st) {
    hipLaunchKernelGGL((moe_choose_kernel<T>), dim3((unsigned)P.n_tokens), dim3(kRouterWaves * 64), 0, st, P);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = gated ? expert_launch<T, W, kUpGated>(P, st) : expert_launch<T, W, kUpRelu>(P, st);
    if (e == hipSuccess) e = expert_launch<T, W, kDown>(P, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((moe_combine_kernel<T>), dim3((unsigned)((P.cout + 1023) / 1024), (unsigned)P.n_tokens), dim3(256), 0, st, P);
    return hipGetLastError();
}

}  // namespace

// The workspace: the choice (where the caller does not take it), the hidden values and the outputs of every slot.
struct MoeSpace { size_t gate, hidden, slots, end; };
static MoeSpace moe_space(const dc_moe& m, int n_tokens) {
    const size_t slots = (size_t)n_tokens * m.top_k;
    MoeSpace s;
    s.gate = align_up(slots * 4, 256);
    s.hidden = 2 * s.gate;
    s.slots = s.hidden + align_up(slots * align_up(m.hidden, 16) * 4, 256);
    s.end = s.slots + align_up(slots * align_up(m.cout, 4) * 4, 256);
    return s;
}
size_t moe_workspace(const dc_moe& m, int n_tokens) { return moe_space(m, n_tokens).end; }

hipError_t launch_moe(const dc_moe& m, const dc_moe_weights& w, const void* in, void* out, int32_t* experts, float* gates, int n_tokens, int dtype,
                      void* ws, hipStream_t st) {
    Moe P;
    const MoeSpace space = moe_space(m, n_tokens);
    unsigned char* const base = static_cast<unsigned char*>(ws);
    P.x = in; P.router = w.router; P.router_bias = w.router_bias;
    P.up = w.up; P.up_scale = w.up_scale; P.up_bias = w.up_bias;
    P.down = w.down; P.down_scale = w.down_scale; P.down_bias = w.down_bias;
    P.out = out;
    P.choice = experts ? experts : reinterpret_cast<int32_t*>(base);
    P.gate = gates ? gates : reinterpret_cast<float*>(base + space.gate);
    P.hidden_out = base + space.hidden;
    P.slot_out = reinterpret_cast<float*>(base + space.slots);
    P.n_tokens = n_tokens; P.experts = m.experts; P.top_k = m.top_k; P.cin = m.cin; P.hidden = m.hidden; P.cout = m.cout;
    P.renormalize = m.renormalize; P.hidden_pad = (int)align_up(m.hidden, 16); P.cout_pad = (int)align_up(m.cout, 4);
    const bool gated = m.act == DC_MOE_GATED;
    if (dtype == DC_BF16) return m.wtype == DC_I8 ? moe_run<uint16_t, int8_t>(P, gated, st) : moe_run<uint16_t, uint16_t>(P, gated, st);
    return m.wtype == DC_I8 ? moe_run<float, int8_t>(P, gated, st) : moe_run<float, float>(P, gated, st);
}

}  // namespace dc

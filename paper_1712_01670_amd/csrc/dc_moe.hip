// A mixture-of-experts layer for a few tokens (a row per video stream): a router chooses top_k of the experts for every token,
// an expert is a pair of fully-connected layers, and the token's output is the sum of its experts', weighted by the router's
// softmax.  What bounds it is the weights of the chosen experts, each of which is read once for every 32 of its tokens in a
// group of 64 tokens (the next group reads them again).  Launches: the choice, the experts' first layers, their second layers,
// the weighted sum; up to 16 tokens the second layers' last workgroups add up, and where the choice is quick every workgroup of
// the first layers makes it for itself: two launches are left.
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
    unsigned char* hidden_out;         // the experts' hidden values, in blocks of 16 slots (Chosen)
    int n_tokens, experts, top_k, cin, hidden, cout, renormalize;
    int group_blocks, cout_pad;        // blocks of a group of tokens; cout rounded up to 4
    int block_rows;                    // rows of a block of hidden values: 16, or 4 / 8 if there are no more tokens
    float* slot_out;                   // [n_tokens * top_k][cout_pad]: the experts' outputs
    int32_t* done;                     // [down_tiles], up to 16 tokens: workgroups of the second layers that have written theirs
    int down_tiles, route;             // route: the first layers' kernel makes the choice itself
};

constexpr int kMoeTokens = 64;         // tokens that share one pass over the weights
constexpr int kMoeWaves = 4;
constexpr int kMoeRouteTokens = 2;     // whose choice the first layers' workgroups make for themselves (a wavefront each)

// 16 bytes of a row, at any address the type allows.
template <typename E>
__device__ __forceinline__ uintx4 load16(const E* p) {
    uintx4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// 16 bytes of a row whose elements begin inside words of 4 bytes: the five words that hold them, put together where they are used
// (loads at such addresses run at less than half the rate: 32 experts, 4 of 2049 -> 2 x 1025 -> 2049 bf16 for 64 tokens took 225 us
// with them, 149 by words; one smaller everywhere 93).  `at` is an address, whose last two bits say where in its word it begins, relative to a base at a word; each
// word read holds a byte that is asked for.
__device__ __forceinline__ uintx4 load_words(const unsigned char* base, uint32_t at) {
    return load16(reinterpret_cast<const uint32_t*>(__builtin_assume_aligned(base + (at & ~3u), 4)));
}
__device__ __forceinline__ uint32_t load_word_behind(const unsigned char* base, uint32_t at) {
    return *reinterpret_cast<const uint32_t*>(base + ((at + 15) & ~3u));
}
__device__ __forceinline__ void shift_words(uintx4& v, uint32_t behind, uint32_t at) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(i < 3 ? v[i + 1] : behind, v[i], at);
}
// The same from element k0 of a row of K, zeros behind its end: what overlaps the end comes from the row's last 16 bytes.
template <typename E>
__device__ __forceinline__ uintx4 load16_end(const E* __restrict__ row, int k0, int K) {
    constexpr int N = 16 / sizeof(E);
    if (k0 + N <= K) return load16(row + k0);
    unsigned long long lo = 0, hi = 0;
    if (k0 < K) {
        if (K >= N) {
            const uintx4 v = load16(row + K - N);
            const int bits = (k0 - (K - N)) * (int)sizeof(E) * 8;      // 8 .. 120
            lo = (unsigned long long)v[1] << 32 | v[0];
            hi = (unsigned long long)v[3] << 32 | v[2];
            if (bits >= 64) { lo = hi >> (bits - 64); hi = 0; }
            else { lo = lo >> bits | hi << (64 - bits); hi >>= bits; }
        } else {
#pragma unroll 1
            for (int e = 0; k0 + e < K; ++e) {
                typename std::conditional<sizeof(E) == 4, uint32_t, typename std::conditional<sizeof(E) == 2, uint16_t, uint8_t>::type>::type u;
                __builtin_memcpy(&u, row + k0 + e, sizeof u);
                const int bit = e * (int)sizeof(E) * 8;
                if (bit < 64) lo |= (unsigned long long)u << bit;
                else hi |= (unsigned long long)u << (bit - 64);
            }
        }
    }
    return uintx4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// A wavefront's operand for 4 * PE values of K, PE of them a lane (16 bytes of weights): one or more fragments of the matrix
// instruction, which takes 8 bf16 or 1 fp32 of a lane.  8-bit integers are exact in either.
template <typename T, typename W>
struct Operand {
    static constexpr int PE = 16 / sizeof(W), V = PE * sizeof(T) / 16;     // V: 16-byte vectors
    uintx4 v[V];
    // of the tokens' own type
    __device__ __forceinline__ void load_end(const T* row, int k0, int K) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = load16_end(row, k0 + i * (16 / (int)sizeof(T)), K);
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

// A value of every lane put together over the wavefront, the result in all of them: within rows of 16 lanes by DPP (a few cycles a
// step where a shuffle through LDS takes sixty), the four rows by scalars.  Always the same order.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <typename F>
__device__ __forceinline__ uint32_t wave_all(uint32_t v, F f) {
    v = f(v, dpp<0xb1>(v));            // lanes 1 apart, 2 apart, then the halves of a row and the row mirrored
    v = f(v, dpp<0x4e>(v));
    v = f(v, dpp<0x141>(v));
    v = f(v, dpp<0x140>(v));
    const auto row = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); };
    return f(f(row(0), row(16)), f(row(32), row(48)));
}
__device__ __forceinline__ float wave_sum(float v) {
    return __uint_as_float(wave_all(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ float wave_max(float v) {       // (a NaN loses)
    return __uint_as_float(wave_all(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
    return wave_all(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
// Sums over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
    auto add = [&](auto ctrl, auto rows) { v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
    using std::integral_constant;
    add(integral_constant<int, 0x111>(), integral_constant<int, 0xf>());       // lanes before in the row
    add(integral_constant<int, 0x112>(), integral_constant<int, 0xf>());
    add(integral_constant<int, 0x114>(), integral_constant<int, 0xf>());
    add(integral_constant<int, 0x118>(), integral_constant<int, 0xf>());
    add(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());       // the row before, for the second and the fourth
    add(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());       // the first two, for the last two
    return v;
}

// ---- the choice ---------------------------------------------------------------------------------------------------------
// Order of the logits as whole numbers: a NaN stands below every number, -inf is 0 and never chosen.
__device__ __forceinline__ uint32_t logit_key(float l) {
    if (l != l) return 1;
    const uint32_t u = __float_as_uint(l + 0.f);     // -0 is 0
    if (u == 0xff800000u) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A wavefront's logits of N experts from e0 on, STEP apart, for a token: the same operations in the same order wherever it is called.
template <typename T, int N, int STEP>
__device__ __forceinline__ void router_logits(const Moe& P, int token, int e0, float* logits) {
    constexpr int VE = 16 / sizeof(T), AT_ONCE = 4;
    const int lane = threadIdx.x & 63;
    const T* const x = static_cast<const T*>(P.x) + (size_t)token * P.cin;
    const T* w[N];
    float sum[N], bias[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = min(e0 + i * STEP, P.experts - 1);
        w[i] = static_cast<const T*>(P.router) + (size_t)e * P.cin;
        bias[i] = P.router_bias ? P.router_bias[e] : 0.f;
        sum[i] = 0.f;
    }
    for (int k0 = lane * VE; k0 < P.cin; k0 += AT_ONCE * 64 * VE) {
        uintx4 xv[AT_ONCE], wv[N][AT_ONCE];
        if (k0 - lane * VE + AT_ONCE * 64 * VE <= P.cin) {
#pragma unroll
            for (int a = 0; a < AT_ONCE; ++a) {
                xv[a] = load16(x + k0 + a * 64 * VE);
#pragma unroll
                for (int i = 0; i < N; ++i) wv[i][a] = load16(w[i] + k0 + a * 64 * VE);
            }
        } else {
#pragma unroll
            for (int a = 0; a < AT_ONCE; ++a) {
                xv[a] = load16_end(x, k0 + a * 64 * VE, P.cin);
#pragma unroll
                for (int i = 0; i < N; ++i) wv[i][a] = load16_end(w[i], k0 + a * 64 * VE, P.cin);
            }
        }
#pragma unroll
        for (int a = 0; a < AT_ONCE; ++a)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if constexpr (sizeof(T) == 4) {
                        sum[i] = fmaf(__uint_as_float(xv[a][d]), __uint_as_float(wv[i][a][d]), sum[i]);
                    } else {
                        sum[i] = fmaf(__uint_as_float(xv[a][d] << 16), __uint_as_float(wv[i][a][d] << 16), sum[i]);
                        sum[i] = fmaf(__uint_as_float(xv[a][d] & 0xffff0000u), __uint_as_float(wv[i][a][d] & 0xffff0000u), sum[i]);
                    }
                }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        sum[i] = wave_sum(sum[i]);
        if (lane == 0 && e0 + i * STEP < P.experts) logits[e0 + i * STEP] = sum[i] + bias[i];
    }
}
// A wavefront's choice for a token: lane j gets choice j and its gate.
__device__ __forceinline__ void choose_experts(const Moe& P, const float* logits, int& expert, float& gate) {
    constexpr int N = kMoeMaxExperts / 64;
    const int lane = threadIdx.x & 63;
    float top = -INFINITY, sum = 0.f;
    uint32_t key[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * 64 + lane;
        key[i] = e < P.experts ? logit_key(logits[e]) : 0;
        if (e < P.experts) top = fmaxf(top, logits[e]);
    }
    top = wave_max(top);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * 64 + lane;
        if (e < P.experts && logits[e] != -INFINITY) sum += expf(logits[e] - top);
    }
    sum = wave_sum(sum);
    float chosen = 0.f;
    expert = -1;
    gate = 0.f;
    for (int j = 0; j < P.top_k; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) best = max(best, key[i]);
        best = wave_umax(best);
        if (best == 0) break;
        int e = -1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const unsigned long long hit = __ballot(key[i] == best);
            if (e < 0 && hit) e = i * 64 + __ffsll(hit) - 1;       // equal: the lowest index
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * 64 + lane == e) key[i] = 0;
        const float g = expf(logits[e] - top) / sum;
        chosen += g;
        if (lane == j) { gate = g; expert = e; }
    }
    if (expert >= 0 && P.renormalize) gate /= chosen;
}

// A workgroup takes a token: its wavefronts deal the experts among themselves, the first one chooses.  Latency bounds it, a trip to memory,
// one to L2 and the sums over a wavefront: 64 tokens of 2048 bf16, 32 experts 6.4 us, 16 of 1024 fp32, 8 experts 4.4 us.
constexpr int kRouterWaves = 16;
template <typename T>
__global__ __launch_bounds__(kRouterWaves * 64) void moe_choose_kernel(Moe P) {
    __shared__ float logits[kMoeMaxExperts];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, token = blockIdx.x;
    for (int e = wave; e < P.experts; e += kRouterWaves) router_logits<T, 1, 1>(P, token, e, logits);
    __syncthreads();
    if (wave != 0) return;
    int expert;
    float gate;
    choose_experts(P, logits, expert, gate);
    if (lane < P.top_k) {
        P.choice[(size_t)token * P.top_k + lane] = expert;
        P.gate[(size_t)token * P.top_k + lane] = gate;
    }
}

// ---- the experts ----------------------------------------------------------------------------------------------------------
// The slots (token * top_k + choice) of a group of kMoeTokens tokens, by expert.  Every workgroup finds its own: the choices are a few
// hundred numbers.  An expert's slots are dealt in parts of 32, a workgroup each; the hidden values of its i-th slot stand in
// row i % 16 of block base + i / 16, base being the blocks of the experts before (a block has fewer rows if there are no more
// tokens: what a wavefront fetches of it is whole).
constexpr int kMoePart = 32;
struct Chosen {
    int count[kMoeMaxExperts];             // slots of an expert
    int choice[kMoeTokens * kMoeMaxTopK];
    int slot[kMoePart];                    // of this workgroup's part
};
__device__ __forceinline__ void count_experts(const Moe& P, Chosen& C, int t0, int n_tok) {
    constexpr int THREADS = kMoeWaves * 64, N = kMoeTokens * kMoeMaxTopK / THREADS;
    const int n = n_tok * P.top_k, tid = threadIdx.x;
    int mine[N];
#pragma unroll
    for (int i = 0; i < N; ++i) mine[i] = tid + i * THREADS < n ? P.choice[(size_t)t0 * P.top_k + tid + i * THREADS] : -1;
    for (int i = tid; i < kMoeMaxExperts; i += THREADS) C.count[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = tid + i * THREADS;
        if (at < n) C.choice[at] = mine[i];
        if (mine[i] >= 0) atomicAdd(&C.count[mine[i]], 1);
    }
    __syncthreads();
}
// The same with the choice made here, by every workgroup for itself (one or two tokens, a wavefront each); the first workgroup
// leaves it in memory.
template <typename T>
__device__ __forceinline__ void choose_and_count(const Moe& P, Chosen& C, float (*logits)[kMoeMaxExperts], bool leave) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < kMoeMaxExperts; i += kMoeWaves * 64) C.count[i] = 0;
    for (int t = 0; t < P.n_tokens; ++t)
        for (int e = wave; e < P.experts; e += 2 * kMoeWaves) router_logits<T, 2, kMoeWaves>(P, t, e, logits[t]);
    __syncthreads();
    if (wave < P.n_tokens) {
        int expert;
        float gate;
        choose_experts(P, logits[wave], expert, gate);
        if (lane < P.top_k) {
            C.choice[wave * P.top_k + lane] = expert;
            if (expert >= 0) atomicAdd(&C.count[expert], 1);
            if (leave) {
                P.choice[wave * P.top_k + lane] = expert;
                P.gate[wave * P.top_k + lane] = gate;
            }
        }
    }
    __syncthreads();
}
// The a-th part: its expert (-1: there are fewer), its place among the expert's parts, the expert's slots and first block.  Every
// wavefront for itself: a lane per expert, sums over the lanes before.
struct Part { int e, place, n, block, all; };      // all: how many parts there are
__device__ __forceinline__ Part find_part(const Moe& P, const Chosen& C, int a) {
    const int lane = threadIdx.x & 63;
    Part part{-1, 0, 0, 0, 0};
    int parts = 0, blocks = 0;                 // of the experts before
    for (int i = 0; i * 64 < P.experts; ++i) {
        const int n = C.count[i * 64 + lane], own = (n + kMoePart - 1) / kMoePart << 16 | (n + 15) / 16;
        const int sum = wave_scan(own);
        const int before = parts + ((sum - own) >> 16);
        const unsigned long long hit = __ballot(a >= before && a < before + (own >> 16));
        if (hit) {
            const int l = __ffsll(hit) - 1;
            part.e = i * 64 + l;
            part.place = a - __builtin_amdgcn_readlane(before, l);
            part.n = __builtin_amdgcn_readlane(n, l);
            part.block = blocks + __builtin_amdgcn_readlane((sum - own) & 0xffff, l);
        }
        const int all = __builtin_amdgcn_readlane(sum, 63);
        parts += all >> 16;
        blocks += all & 0xffff;
    }
    part.all = parts;
    return part;
}
// How many parts there are.
__device__ __forceinline__ int count_parts(const Moe& P, const Chosen& C) {
    int parts = 0;
    for (int i = 0; i * 64 < P.experts; ++i) parts += __builtin_amdgcn_readlane(wave_scan((C.count[i * 64 + (threadIdx.x & 63)] + kMoePart - 1) / kMoePart), 63);
    return parts;
}
// Slots of the part in order, by the first wavefront, a lane per token.
__device__ __forceinline__ void list_slots(const Moe& P, Chosen& C, const Part& part, int t0, int n_tok) {
    if (threadIdx.x < 64) {
        int at = -1;
        if ((int)threadIdx.x < n_tok)
            for (int j = 0; j < P.top_k; ++j)
                if (C.choice[threadIdx.x * P.top_k + j] == part.e) at = (t0 + threadIdx.x) * P.top_k + j;
        const unsigned long long m = __ballot(at >= 0);
        const int i = __popcll(m & ((1ull << threadIdx.x) - 1)) - part.place * kMoePart;
        if (at >= 0 && i >= 0 && i < kMoePart) C.slot[i] = at;
    }
    __syncthreads();
}

// Outputs of a slot.  SHARED: workgroups of the same launch, on whichever XCD, write and read them: then by atomic operations of the
// GPU's scope, which go past the XCDs' own caches (a fence would write those back and drop what they hold: with one a
// workgroup the second layers of 32 experts took 194 us instead of 33).
template <bool SHARED>
__device__ __forceinline__ void put_slot(float* p, const floatx4& v) {
    if constexpr (SHARED) {
        unsigned long long u[2];
        __builtin_memcpy(u, &v, 16);
#pragma unroll
        for (int i = 0; i < 2; ++i) __hip_atomic_store(reinterpret_cast<unsigned long long*>(p) + i, u[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else {
        *reinterpret_cast<floatx4*>(p) = v;
    }
}
template <bool SHARED>
__device__ __forceinline__ floatx4 get_slot(const float* p) {
    if constexpr (!SHARED) return *reinterpret_cast<const floatx4*>(p);
    unsigned long long u[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) u[i] = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    floatx4 v;
    __builtin_memcpy(&v, u, 16);
    return v;
}
// out[token] = sum over its choices, in their order, of gate * the slot's output; four channels.  `choice`: the token's.
template <typename T, bool SHARED>
__device__ __forceinline__ void combine(const Moe& P, const int* choice, int token, int c) {
    floatx4 sum{0.f, 0.f, 0.f, 0.f};
    const size_t slot0 = (size_t)token * P.top_k;
    for (int j0 = 0; j0 < P.top_k; j0 += 4) {          // four outputs on their way together
        floatx4 y[4];
        float gate[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = min(j0 + j, P.top_k - 1);
            y[j] = get_slot<SHARED>(P.slot_out + (slot0 + at) * P.cout_pad + c);
            gate[j] = P.gate[slot0 + at];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j0 + j < P.top_k && choice[j0 + j] >= 0)           // (an empty place has no output)
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[q] = fmaf(gate[j], y[j][q], sum[q]);
    }
    T* const out = static_cast<T*>(P.out) + (size_t)token * P.cout + c;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (c + q < P.cout) store(out + q, sum[q]);
}
// More than 16 tokens: a launch of its own (64 tokens x 4 choices of 2048 4.7 us, of which 2.7 are any launch's; as part of the second layers
// it would take an atomic per workgroup and token group).
template <typename T>
__global__ __launch_bounds__(256) void moe_combine_kernel(Moe P) {
    const int c = (blockIdx.x * 256 + threadIdx.x) * 4, token = blockIdx.y;
    if (c < P.cout) combine<T, false>(P, P.choice + (size_t)token * P.top_k, token, c);
}

// The product of R tiles of 16 channels of an expert (gated: R / 2 in either half) with a part of its slots: relu or gate of
// the first layer into the hidden values, or the second layer into the slots' outputs.  The weights are what has to come from
// memory, once: they go straight into operands (16 rows of 64 bytes an instruction), two pieces of a wavefront
// ahead, both halves of a cache line one after the other (reading 268 MB that way takes 51 us, a half of all lines and then the
// other 62; four rows of 256 bytes 47).  Every wavefront takes a run of K, of whole cache lines; their sums are added through LDS in a
// fixed order.  The tokens' rows come from L2, once for R tiles of weights: a row of a fragment costs the CU a look-up for
// every 16 bytes, as a row of weights does, so R is large where there are workgroups enough.  The hidden values lie in the order
// of the second layer's fragments, 1 KiB a look-up of 16, fp32 or as two bf16 numbers each (the value's rounding and what
// that leaves), so that the second product sees 16 bits of them: the layer's output is rounded once, as if they were fp32.
// Measured, first and second layers (rate of the weights): 64 tokens, 32 experts, 4 of 2048 -> 2 x 1024 -> 2048 bf16 51 us (5.2 TB/s)
// and 29 (4.6); 8 experts, 2 of 4096 -> 2 x 8192 -> 4096 in 8 bits 113 (4.7) and 73 (3.7: the hidden values, twice 16 bits, are four times
// a row of weights); 16 tokens, 8 experts, 2 of 1024 -> 2048 -> 1024 fp32 17 and 17 (4.0); one token, 2 of 2048 -> 2 x 4096 -> 2048 bf16 17
// (3.9) and 13 (2.5): 5 us of each are the start of the kernel, the first trip to memory and the sums' way out.
__device__ __forceinline__ int opaque(int v) {      // a value the optimiser computes nothing from ahead of time
    asm volatile("" : "+v"(v));
    return v;
}
enum { kUpRelu = 0, kUpGated = 1, kDown = 2 };
template <typename T, typename W, int KIND, int R, int MOST, bool ODD>      // ODD: rows that begin inside words of 4 bytes
__global__ __launch_bounds__(kMoeWaves * 64) void moe_expert_kernel(Moe P) {
    typedef Operand<T, W> Op;
    constexpr int PE = Op::PE, V = Op::V, HALVES = KIND == kUpGated ? 2 : 1, CT = R / HALVES, PLANES = sizeof(T) == 2 ? 2 : 1;
    constexpr bool DOWN = KIND == kDown, TWO = DOWN && PLANES == 2, ADDS = DOWN && MOST == 1;      // ADDS: the slots' outputs up, too
    constexpr bool ODD_X = ODD && !DOWN && sizeof(T) == 2;
    __shared__ Chosen C;
    __shared__ floatx4 red[kMoeWaves][R][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int channels = DOWN ? P.cout : P.hidden, K = DOWN ? P.hidden : P.cin;
    const int t0 = blockIdx.z * kMoeTokens, n_tok = min(kMoeTokens, P.n_tokens - t0);
    const int pieces = (K + 4 * PE - 1) / (4 * PE), whole = K / (4 * PE), hidden_pieces = (P.hidden + 4 * PE - 1) / (4 * PE);
    const int piece_bytes = P.block_rows * (V * 64);       // of a block of hidden values
    if constexpr (DOWN || MOST > 1) {
        count_experts(P, C, t0, n_tok);
    } else {
        if (P.route) choose_and_count<T>(P, C, reinterpret_cast<float(*)[kMoeMaxExperts]>(&red[0][0][0]), blockIdx.x == 0 && blockIdx.y == 0);
        else count_experts(P, C, t0, n_tok);
    }
    int tile = blockIdx.x, at = blockIdx.y;
    if constexpr (DOWN && MOST > 1) {      // an XCD (workgroup number modulo 8) takes a run of the tiles, so that few of them fetch an expert's hidden values
        const int all = count_parts(P, C) * gridDim.x, number = blockIdx.y * gridDim.x + blockIdx.x;
        const int xcd = number & 7, j = number >> 3, per = all >> 3, more = all & 7;
        if (j >= per + (xcd < more)) return;
        const int i = xcd * per + min(xcd, more) + j;
        at = i / gridDim.x;
        tile = i % gridDim.x;
    }
    const Part part = find_part(P, C, at);
    const int e = part.e, o0 = tile * (CT * 16);
    auto add_up = [&]() {
        for (int i = tid; i < n_tok * (CT * 4); i += kMoeWaves * 64) {
            const int t = i / (CT * 4), c = o0 + i % (CT * 4) * 4;
            if (c < P.cout) combine<T, true>(P, C.choice + t * P.top_k, t0 + t, c);
        }
    };
    if constexpr (ADDS) {
        if (part.all == 0 && blockIdx.y == 0) add_up();    // no token has an expert
    }
    if constexpr (!DOWN && MOST == 1) {
        if (blockIdx.x == 0 && blockIdx.y == 0)
            for (int i = tid; i < P.down_tiles; i += kMoeWaves * 64) P.done[i] = 0;
    }
    if (e < 0) return;
    // Addresses are a uniform base and 32 bits a lane, so that what is ahead costs no registers but its own.  Tile r: half r / CT,
    // channels 16 (r % CT) on; past the end the last channel again (also where a tile starts there: hidden values are made up to
    // whole pieces).
    const int row0 = min(o0, channels - 1);
    const unsigned char* wbase[HALVES];
    uint32_t wat[ODD ? R : CT];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        wbase[h] = reinterpret_cast<const unsigned char*>(static_cast<const W*>(DOWN ? P.down : P.up) + (((size_t)e * HALVES + h) * channels + row0) * K);
        if (ODD || h == 0)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                wat[h * CT + c] = (uint32_t)(min(o0 + c * 16 + l16, channels - 1) - row0) * (uint32_t)(K * sizeof(W)) + g * 16;
                if constexpr (ODD) wat[h * CT + c] += reinterpret_cast<uintptr_t>(wbase[h]) & 3;
            }
        if constexpr (ODD) wbase[h] -= reinterpret_cast<uintptr_t>(wbase[h]) & 3;
    }
    const int share = ((whole + 1) / 2 + kMoeWaves - 1) / kMoeWaves * 2, first = wave * share, end = min(whole, first + share);      // this wavefront's pieces
    uintx4 w[4][R];
    uint32_t w_behind[4][ODD ? R : 1];
    auto fetch_w = [&](int d, int p) {                     // two pieces: a cache line of every row
        if (p < end) {
            const uint32_t at = p * 64, at1 = p + 1 < end ? at + 64 : at;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (ODD) {
                    w[d][r] = load_words(wbase[r / CT] + at, wat[r]);
                    w[d + 1][r] = load_words(wbase[r / CT] + at1, wat[r]);
                    w_behind[d][r] = load_word_behind(wbase[r / CT] + at, wat[r]);
                    w_behind[d + 1][r] = load_word_behind(wbase[r / CT] + at1, wat[r]);
                } else {
                    w[d][r] = load16(wbase[r / CT] + at + wat[r % CT]);
                    w[d + 1][r] = load16(wbase[r / CT] + at1 + wat[r % CT]);
                }
            }
        }
    };
    fetch_w(0, first);
    floatx4 scale[HALVES], bias[HALVES];                   // of the channels that this wavefront finishes
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            scale[h][q] = 1.f;
            bias[h][q] = 0.f;
            if (wave < CT) {
                const size_t c = ((size_t)e * HALVES + h) * channels + min(o0 + wave * 16 + g * 4 + q, channels - 1);
                if constexpr (sizeof(W) == 1) scale[h][q] = (DOWN ? P.down_scale : P.up_scale)[c];
                const float* const b = DOWN ? P.down_bias : P.up_bias;
                if (b) bias[h][q] = b[c];
            }
        }
    list_slots(P, C, part, t0, n_tok);                     // (while the first weights travel)
    const int n = min(kMoePart, part.n - part.place * kMoePart);
    unsigned char* const tiles = P.hidden_out + ((size_t)blockIdx.z * P.group_blocks + part.block + part.place * (kMoePart / 16)) * PLANES * hidden_pieces * piece_bytes;
    auto product = [&](auto blocks) {                      // of 16 slots
        constexpr int NB = decltype(blocks)::value;
        const unsigned char* xbase[DOWN ? NB : 1];
        uint32_t xat[DOWN ? 1 : NB];
        if constexpr (DOWN) {
            xat[0] = (g * P.block_rows + (NB == 1 ? min(l16, n - 1) : l16)) * 16;      // (rows that are not there repeat the last one)
#pragma unroll
            for (int j = 0; j < NB; ++j) xbase[j] = tiles + (size_t)j * PLANES * hidden_pieces * piece_bytes;
        } else {
            const uint32_t into = ODD_X ? reinterpret_cast<uintptr_t>(P.x) & 3 : 0;
            xbase[0] = static_cast<const unsigned char*>(P.x) - into;
#pragma unroll
            for (int j = 0; j < NB; ++j) xat[j] = (uint32_t)(C.slot[min(j * 16 + l16, n - 1)] / P.top_k) * (uint32_t)(P.cin * sizeof(T)) + into;
        }
        constexpr int XRING = NB == 1 ? 4 : 2;             // rows of one block travel by pairs of pieces, too, of two a piece ahead
        Op x[XRING][NB], low[XRING][TWO ? NB : 1];
        uint32_t x_behind[XRING][ODD_X ? NB : 1];
        auto fetch_x = [&](int b, int p, bool end = false, int k0 = 0) {
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if constexpr (DOWN) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const unsigned char* const from = xbase[j] + (uint32_t)(p * piece_bytes + v * (piece_bytes / V));
                        x[b][j].v[v] = load16(from + xat[0]);
                        if constexpr (TWO) low[b][j].v[v] = load16(from + (uint32_t)(hidden_pieces * piece_bytes) + xat[0]);
                    }
                } else if (end) {
                    x[b][j].load_end(reinterpret_cast<const T*>(xbase[0] + xat[j]), k0, K);
                } else if constexpr (ODD_X) {
#pragma unroll
                    for (int v = 0; v < V; ++v) x[b][j].v[v] = load_words(xbase[0] + (uint32_t)(p * (V * 64) + v * 16), xat[j] + g * (V * 16));
                    x_behind[b][j] = load_word_behind(xbase[0] + (uint32_t)(p * (V * 64) + (V - 1) * 16), xat[j] + g * (V * 16));
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v) x[b][j].v[v] = load16(xbase[0] + (uint32_t)(p * (V * 64) + v * 16) + (xat[j] + g * (V * 16)));
                }
            }
        };
        floatx4 acc[R][NB];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[r][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        auto multiply = [&](int d, int b, bool end = false) {
            if constexpr (ODD_X)
                if (!end)
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int v = 0; v < V; ++v) shift_words(x[b][j].v[v], v + 1 < V ? x[b][j].v[v + 1 < V ? v + 1 : v][0] : x_behind[b][j], xat[j]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uintx4 raw = w[d][r];
                asm volatile("" : "+v"(raw));                  // (converted here, not where it is loaded: the ring holds bytes)
                if constexpr (ODD)
                    if (!end) shift_words(raw, w_behind[d][r], wat[r]);
                const Op o(raw);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    mma(o, x[b][j], acc[r][j]);
                    if constexpr (TWO) mma(o, low[b][j], acc[r][j]);
                }
            }
        };
        auto fetch_xs = [&](int d, int p) {                // XRING / 2 pieces
#pragma unroll
            for (int i = 0; i < XRING / 2; ++i)
                if (p + i < end) fetch_x((d + i) % XRING, p + i);
        };
        fetch_xs(0, first);
        for (int p = first; p < end; p += 4) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {                  // (loads come back in order: the rows before the weights further ahead)
                if (XRING == 2 || d % 2 == 0) fetch_xs(d + XRING / 2, p + d + XRING / 2);
                if (d % 2 == 0) fetch_w((d + 2) & 3, p + d + 2);
                __builtin_amdgcn_sched_barrier(0);
                if (p + d < end) multiply(d, d % XRING);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (pieces > whole && wave == kMoeWaves - 1) {         // the piece that K ends in
            const int k0 = opaque(whole * (4 * PE) + g * PE);
#pragma unroll
            for (int r = 0; r < R; ++r) w[0][r] = load16_end(reinterpret_cast<const W*>(wbase[r / CT] + (wat[ODD ? r : r % CT] - g * 16)), k0, K);
            fetch_x(0, whole, true, k0);
            multiply(0, 0, true);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) red[wave][r][lane] = acc[r][j];
            __syncthreads();
            const int i = j * 16 + l16, ct = wave;      // wavefront ct: tile ct of the channels
            if (ct >= CT || i >= n) continue;
            const int slot = C.slot[i], c0 = opaque(o0 + ct * 16 + g * 4);       // (what follows from it is not worth registers in the loop)
            floatx4 sum[HALVES];
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                sum[h] = red[0][h * CT + ct][lane];
#pragma unroll
                for (int v = 1; v < kMoeWaves; ++v) sum[h] += red[v][h * CT + ct][lane];
#pragma unroll
                for (int q = 0; q < 4; ++q) sum[h][q] = fmaf(sum[h][q], scale[h][q], bias[h][q]);
            }
            if constexpr (DOWN) {
                if (c0 < P.cout_pad) put_slot<ADDS>(P.slot_out + (size_t)slot * P.cout_pad + c0, sum[0]);
            } else {
                if (c0 >= hidden_pieces * 4 * PE) continue;
                T high[4], rest[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float u = sum[0][q];
                    float v;
                    if constexpr (KIND == kUpGated) v = u / (1.f + expf(-u)) * sum[HALVES - 1][q];
                    else v = u > 0.f || u != u ? u : 0.f;
                    if (c0 + q >= P.hidden) v = 0.f;           // behind the last channel the second layer multiplies zeros
                    store(&high[q], v);
                    if constexpr (PLANES == 2)
                        if (fabsf(v) < INFINITY && (high[q] & 0x7fff) == 0x7f80) --high[q];      // (a number that rounds to infinity: the largest below)
                    const float h = to_float(high[q]);
                    store(&rest[q], fabsf(h) < INFINITY || h != h ? v - h : 0.f);
                }
                // channel c0 is element c0 % PE of lane group c0 / PE % 4 of piece c0 / (4 PE)
                constexpr int VE = 16 / sizeof(T);
                unsigned char* const to = tiles + (size_t)j * PLANES * hidden_pieces * piece_bytes + (size_t)(c0 / (4 * PE)) * piece_bytes +
                                          c0 % PE / VE * (piece_bytes / V) + (c0 / PE % 4 * P.block_rows + l16) * 16 + c0 % VE * sizeof(T);
                __builtin_memcpy(__builtin_assume_aligned(to, 4 * sizeof(T)), high, sizeof high);
                if constexpr (PLANES == 2) __builtin_memcpy(__builtin_assume_aligned(to + (size_t)hidden_pieces * piece_bytes, 4 * sizeof(T)), rest, sizeof rest);
            }
        }
    };
    if (MOST == 1 || n <= 16) product(std::integral_constant<int, 1>());
    else product(std::integral_constant<int, 2>());
    if constexpr (ADDS) {
        // The workgroup that comes last for these channels adds up; nothing waits for another.
        __shared__ int last;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's outputs have arrived
        __syncthreads();
        if (tid == 0) last = __hip_atomic_fetch_add(P.done + blockIdx.x, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == part.all - 1;
        __syncthreads();
        if (last) add_up();
    }
}

template <typename T, typename W, int KIND, int R>
hipError_t expert_launch_as(const Moe& P, unsigned tiles, unsigned parts, bool odd, hipStream_t st) {
    const dim3 grid(tiles, parts, (unsigned)((P.n_tokens + kMoeTokens - 1) / kMoeTokens)), block(kMoeWaves * 64);
    auto go = [&](auto is_odd) {
        constexpr bool ODD = decltype(is_odd)::value;
        if (P.n_tokens <= 16) hipLaunchKernelGGL((moe_expert_kernel<T, W, KIND, R, 1, ODD>), grid, block, 0, st, P);
        else hipLaunchKernelGGL((moe_expert_kernel<T, W, KIND, R, 2, ODD>), grid, block, 0, st, P);
        return hipGetLastError();
    };
    if constexpr (sizeof(W) < 4)
        if (odd) return go(std::true_type());
    return go(std::false_type());
}
// Tiles of channels a workgroup: more of them share a fragment of the rows, fewer give more workgroups.  Few tokens have one fragment
// and want four workgroups a CU (us, four tiles -> fewer: 1024 -> 2048 -> 1024 fp32 16 rows 22.7 + 25.8 -> 20.7 + 22.8), more want the sharing
// as long as there is one for every CU (8192 -> 4096 in 8 bits 64 rows 80 -> 95).
struct Shape { int tiles; unsigned wgs; };
Shape shape_of(const Moe& P, int channels, int halves, unsigned parts) {
    const unsigned want = P.n_tokens <= 16 ? 1024 : 256;
    for (int r = 4; r >= halves; r >>= 1) {
        const unsigned wgs = (unsigned)(channels + 16 * r / halves - 1) / (16 * r / halves);
        if (wgs * parts >= want || r == halves) return Shape{r, wgs};
    }
    return Shape{halves, 0};       // (not reached)
}
template <typename T, typename W, int KIND>
hipError_t expert_launch(const Moe& P, const Shape& s, unsigned parts, hipStream_t st) {
    const size_t row = (KIND == kDown ? P.hidden : P.cin) * sizeof(W);
    bool odd = (reinterpret_cast<uintptr_t>(KIND == kDown ? P.down : P.up) | row) & 3;
    if (KIND != kDown) odd = odd || ((reinterpret_cast<uintptr_t>(P.x) | P.cin * sizeof(T)) & 3);
    if (s.tiles == 4) return expert_launch_as<T, W, KIND, 4>(P, s.wgs, parts, odd, st);
    if constexpr (KIND != kUpGated)
        if (s.tiles == 1) return expert_launch_as<T, W, KIND, 1>(P, s.wgs, parts, odd, st);
    return expert_launch_as<T, W, KIND, 2>(P, s.wgs, parts, odd, st);
}

template <typename T, typename W>
hipError_t moe_run(Moe& P, bool gated, hipStream_t st) {
    const int slots = std::min(P.n_tokens, kMoeTokens) * P.top_k;
    const unsigned parts = (unsigned)(std::min(P.experts, slots) + (P.n_tokens > kMoePart ? slots / (kMoePart + 1) : 0));      // at most
    constexpr int kPiece = 64 / sizeof(W);
    const Shape up = shape_of(P, (P.hidden + kPiece - 1) / kPiece * kPiece, gated ? 2 : 1, parts);       // (whole pieces of hidden values)
    const Shape down = shape_of(P, P.cout, 1, parts);
    P.down_tiles = (int)down.wgs;
    // The choice within the first layers saves a launch, but every workgroup reads the whole router and adds up n_tokens * experts logits
    // (us a call, a launch of its own -> within; 1024 -> 2 x 512 -> 1024 bf16, 2 chosen): one token 8 experts 14.9 -> 13.4, 16 15.7 -> 15.3, 32
    // 16.9 -> 18.1; two tokens 8 experts 15.4 -> 15.4, 16 16.4 -> 19.3; four tokens 4 experts 15.4 -> 18.2.  Two tokens and 4 experts:
    // rows of 4096 21.9 -> 22.3, of 8192 30.9 -> 33.3; one token and 8 experts, of 8192 30.5 -> 29.3.
    P.route = P.n_tokens <= kMoeRouteTokens && P.n_tokens * P.experts <= 16 && P.n_tokens * P.cin * (int)sizeof(T) <= 16384;
    hipError_t e = hipSuccess;
    if (!P.route) {
        hipLaunchKernelGGL((moe_choose_kernel<T>), dim3((unsigned)P.n_tokens), dim3(kRouterWaves * 64), 0, st, P);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = gated ? expert_launch<T, W, kUpGated>(P, up, parts, st) : expert_launch<T, W, kUpRelu>(P, up, parts, st);
    if (e == hipSuccess) e = expert_launch<T, W, kDown>(P, down, parts, st);
    if (e != hipSuccess || P.n_tokens <= 16) return e;
    hipLaunchKernelGGL((moe_combine_kernel<T>), dim3((unsigned)((P.cout + 1023) / 1024), (unsigned)P.n_tokens), dim3(256), 0, st, P);
    return hipGetLastError();
}

}  // namespace

// The workspace: the choice (where the caller does not take it), the hidden values and the outputs of every slot.
struct MoeSpace { size_t gate, hidden, slots, done, end; };
static int block_rows(int n_tokens) { return n_tokens <= 4 ? 4 : n_tokens <= 8 ? 8 : 16; }
static size_t group_blocks(const dc_moe& m, int n_tokens) {
    const int tokens = std::min(n_tokens, kMoeTokens);
    return ((size_t)tokens * m.top_k + 15 * (size_t)std::min(m.experts, tokens * m.top_k)) / 16;
}
static MoeSpace moe_space(const dc_moe& m, int n_tokens) {
    const size_t slots = (size_t)n_tokens * m.top_k;
    MoeSpace s;
    s.gate = align_up(slots * 4, 256);
    s.hidden = 2 * s.gate;
    // (rows of the type's own size or two of half of it; an expert's last block is not full)
    s.slots = s.hidden + ((size_t)n_tokens + kMoeTokens - 1) / kMoeTokens * group_blocks(m, n_tokens) * block_rows(n_tokens) * align_up(m.hidden, 64) * 4;
    s.done = s.slots + align_up(slots * align_up(m.cout, 4) * 4, 256);
    s.end = s.done + align_up((size_t)((m.cout + 15) / 16) * 4, 256);
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
    P.done = reinterpret_cast<int32_t*>(base + space.done);
    P.n_tokens = n_tokens; P.experts = m.experts; P.top_k = m.top_k; P.cin = m.cin; P.hidden = m.hidden; P.cout = m.cout;
    P.renormalize = m.renormalize; P.group_blocks = (int)group_blocks(m, n_tokens); P.block_rows = block_rows(n_tokens); P.cout_pad = (int)align_up(m.cout, 4);
    const bool gated = m.act == DC_MOE_GATED;
    if (dtype == DC_BF16) return m.wtype == DC_I8 ? moe_run<uint16_t, int8_t>(P, gated, st) : moe_run<uint16_t, uint16_t>(P, gated, st);
    return m.wtype == DC_I8 ? moe_run<float, int8_t>(P, gated, st) : moe_run<float, float>(P, gated, st);
}

}  // namespace dc

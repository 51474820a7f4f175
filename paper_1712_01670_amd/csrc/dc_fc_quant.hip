// Fully-connected layers in 8-bit integers.  A row (a token, a pixel, a stream's features) is rounded to 8 bits with a scale of
// its own, the weights have a scale per output channel, so that
//   out[r][o] = act(sx[r] sw[o] sum_k q[r][k] w[o][k] + bias[o])
// with an integer sum that is exact whatever its order: results do not depend on which kernel runs, on how K is split or on
// how many rows a call has.
#include <hip/hip_bf16.h>

#include <algorithm>
#include <atomic>

#include "dc_fc_quant_plan.h"
#include "dc_internal.h"

namespace dc {
namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx4_any __attribute__((ext_vector_type(4), aligned(1)));      // 16 bytes at any address
typedef float floatx4 __attribute__((ext_vector_type(4)));

// ---- rounding rows to 8 bits ------------------------------------------------------------------------------------------
// scale = max |x| / 127 in fp32, q = x / scale rounded half to even: of the exact quotient, not of its fp32 rounding, so that
// any other implementation of the definition agrees.  The remainder x - q s of a quotient that is off by one at most is exact
// in one fma (x and s have 24 bits each and the quotient 7), and deciding by it costs two comparisons where the division's
// correction would cost five instructions.  A row that holds a NaN or an infinity has the scale NaN (and zeros); a row of
// zeros has the scale 0.
__device__ __forceinline__ int quotient8(float x, float s, float inv) {
    float q = rintf(x * inv);
    const float r2 = 2.f * fmaf(-q, s, x);
    const bool odd = ((int)q & 1) != 0;
    if (r2 > s || (r2 == s && odd)) q += 1.f;
    else if (r2 < -s || (r2 == -s && odd)) q -= 1.f;
    return (int)fminf(fmaxf(q, -127.f), 127.f);      // (a scale among the subnormal numbers is coarse: more than 127 of it fit)
}
// N of them, as bytes.  x times 1 / s is within 8e-6 of the quotient (1 / s is off by half a step, the product goes into the sum
// unrounded, and the quotient is 127 at most), so its nearest integer is the right one unless it lies that close to the border:
// then, for one vector of a wavefront in a hundred, the exact form above decides.  Adding 1.5 * 2^23 rounds to an integer, whose
// low byte is the result.
constexpr float kRound = 12582912.f;
template <int N>
__device__ __forceinline__ void quotients8(const float (&x)[N], float s, float inv, uint32_t (&v)[N / 4]) {
    uint32_t r[N];
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float t = fmaf(x[e], inv, kRound);
        r[e] = __float_as_uint(t);
        off = fmaxf(off, fabsf(fmaf(x[e], inv, kRound - t)));
    }
    if (!(off < 0.49999f && s >= 0x1p-100f)) {
        const float up = s < 0x1p-100f ? 0x1p64f : 1.f;      // keeps 1 / s finite; a power of two changes no quotient
        const float su = s * up, iu = 1.f / su;
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = (uint32_t)quotient8(x[e] * up, su, iu);
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(r[4 * i + 1], r[4 * i], 0x0c0c0400u), hi = __builtin_amdgcn_perm(r[4 * i + 3], r[4 * i + 2], 0x0c0c0400u);
        v[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
}

// 16 bytes of a row as fp32, at any address its type allows; zeros behind the row's end.
template <typename T>
struct RowVec;
template <>
struct RowVec<float> {
    static constexpr int N = 4;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void load(const float* p, float (&f)[4]) {
        const any v = *reinterpret_cast<const any*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
    }
};
template <>
struct RowVec<__hip_bfloat16> {
    static constexpr int N = 8;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ float one(const __hip_bfloat16* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ void load(const __hip_bfloat16* p, float (&f)[8]) {
        const any v = *reinterpret_cast<const any*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = __uint_as_float(v[e] << 16);
            f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        }
    }
};
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* row, int k0, int K, float (&f)[N]) {
    if (k0 + N <= K) {
        RowVec<T>::load(row + k0, f);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = k0 + e < K ? RowVec<T>::one(row + k0 + e) : 0.f;
    }
}

// What the bits of a row's largest |x| make of it.
struct RowScale {
    float scale, s, inv;
    bool zero;
    __device__ __forceinline__ explicit RowScale(uint32_t top) {
        const bool bad = top >= 0x7f800000u;
        s = __uint_as_float(top) / 127.f;
        scale = bad ? __uint_as_float(0x7fc00000u) : s;
        zero = bad || !(s > 0.f);
        inv = 1.f / s;
    }
};

// Where a row's bytes go: [n_rows][stride], `width` of them (zeros behind K); or tiles of 16 rows x 64 bytes in the order of a
// fragment's lanes (lane l: row l % 16, bytes 16 (l / 16) on), 1 KiB in one piece, tile (i, j) being number i * n_tiles + j.
// The counters that the product behind it wants at zero come along.
struct Rows8 { int8_t* q; size_t stride; int width; int32_t* zero = nullptr; int zeros = 0; };
__device__ __forceinline__ size_t tile_offset(size_t row, int k0, int n_tiles) {
    return ((row >> 4) * n_tiles + (k0 >> 6)) * 1024 + ((k0 >> 4) & 3) * 256 + (row & 15) * 16 + (k0 & 15);
}
template <bool TILED, int N>
__device__ __forceinline__ void store8(const Rows8& to, size_t row, int k0, const uint32_t (&v)[N / 4]) {
    typedef uint32_t any __attribute__((ext_vector_type(N / 4), aligned(TILED ? N : 1)));
    any w;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = v[i];
    if constexpr (TILED) {
        *reinterpret_cast<any*>(to.q + tile_offset(row, k0, to.width >> 6)) = w;
    } else if (k0 + N <= to.width) {
        *reinterpret_cast<any*>(to.q + row * to.stride + k0) = w;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (k0 + e < to.width) to.q[row * to.stride + k0 + e] = (int8_t)(v[e >> 2] >> (8 * (e & 3)));
    }
}

// LANES threads share a row, a vector each and LANES vectors further the next.  CH > 0: they hold the row in registers, so it is
// read once; CH == 0: a row that is too long for that is read twice, the second time from the cache.  Memory bounds it where there are many
// rows: 16384 x 4096 bf16 46.7 us (201 MB, 4.3 TB/s), 12544 x 1024 14.6 us from memory, 7.9 from the cache; 3 to 5 us, the way
// through the row's maximum, where there are few.
template <typename T, int LANES, int CH, bool TILED>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void quantize_rows_kernel(const T* __restrict__ x, size_t n_rows, int K, Rows8 to,
                                                                                  float* __restrict__ scales) {
    constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES, N = RowVec<T>::N;
    const int tid = threadIdx.x, part = tid % LANES;
    const size_t row = (size_t)blockIdx.x * ROWS + tid / LANES;
    const bool live = row < n_rows;
    if (blockIdx.x == 0)
        for (int i = tid; i < to.zeros; i += THREADS) to.zero[i] = 0;
    const T* const xr = x + (live ? row : 0) * K;
    const int vecs = live ? (to.width + N - 1) / N : 0;
    float f[CH ? CH : 1][N];
    uint32_t top = 0;                                // the largest |x|: as whole numbers, infinities and NaN come out on top
    auto look = [&](const float (&v)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    };
    if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * LANES + part < vecs) {
                load_row(xr, (c * LANES + part) * N, K, f[c]);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) f[c][e] = 0.f;
            }
#pragma unroll
        for (int c = 0; c < CH; ++c) look(f[c]);
    } else {
        for (int i = part; i < vecs; i += LANES) {
            load_row(xr, i * N, K, f[0]);
            look(f[0]);
        }
    }
#pragma unroll
    for (int d = (LANES < 64 ? LANES : 64) / 2; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if constexpr (LANES > 64) {
        __shared__ uint32_t tops[THREADS / 64];
        if ((tid & 63) == 0) tops[tid >> 6] = top;
        __syncthreads();
        const int first = tid / LANES * (LANES / 64);
#pragma unroll
        for (int i = 0; i < LANES / 64; ++i) top = max(top, tops[first + i]);
    }
    if (!live) return;
    const RowScale s(top);
    if (part == 0) scales[row] = s.scale;
    auto put = [&](int i, const float (&v)[N]) {
        uint32_t w[N / 4] = {};
        if (!s.zero) quotients8(v, s.s, s.inv, w);
        store8<TILED, N>(to, row, i * N, w);
    };
    if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * LANES + part < vecs) put(c * LANES + part, f[c]);
    } else {
        for (int i = part; i < vecs; i += LANES) {
            load_row(xr, i * N, K, f[0]);
            put(i, f[0]);
        }
    }
}

template <typename T, bool TILED>
hipError_t quantize(const T* x, size_t n_rows, int K, const Rows8& to, float* scales, hipStream_t st) {
    auto go = [&](auto lanes, auto ch) {
        constexpr int LANES = decltype(lanes)::value, CH = decltype(ch)::value, THREADS = LANES > 256 ? LANES : 256;
        constexpr size_t kMost = 1 << 20;            // rows of a launch: its threads are counted in 32 bits
        for (size_t r = 0; r < n_rows; r += kMost) {
            const size_t n = std::min(kMost, n_rows - r), wgs = (n + THREADS / LANES - 1) / (THREADS / LANES);
            hipLaunchKernelGGL((quantize_rows_kernel<T, LANES, CH, TILED>), dim3((unsigned)wgs), dim3(THREADS), 0, st, x + r * K, n, K,
                               Rows8{to.q + r * to.stride, to.stride, to.width, to.zero, to.zeros}, scales + r);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    using std::integral_constant;
    const int vecs = (to.width + RowVec<T>::N - 1) / RowVec<T>::N;
    // a vector or two a thread is the shortest way through a row; many rows want up to four, whose loads travel together, and few
    // lanes, whose sums are cheap (12544 rows of 1024 bf16: 16 x 8 8.7 us, 32 x 4 7.9, 128 x 4 11.0, 256 x 1 12.4; 50176 of 256: 16 x 4
    // 8.4, 64 x 2 15.4, 256 x 1 33.5)
    if (n_rows < 2048) {
        if (vecs <= 128) return go(integral_constant<int, 64>(), integral_constant<int, 2>());
        if (vecs <= 512) return go(integral_constant<int, 256>(), integral_constant<int, 2>());
    } else if constexpr (!TILED) {
        if (vecs <= 64) return go(integral_constant<int, 16>(), integral_constant<int, 4>());
        if (vecs <= 128) return go(integral_constant<int, 32>(), integral_constant<int, 4>());
        if (vecs <= 256) return go(integral_constant<int, 64>(), integral_constant<int, 4>());
        if (vecs <= 512) return go(integral_constant<int, 128>(), integral_constant<int, 4>());
        if (vecs <= 1024) return go(integral_constant<int, 256>(), integral_constant<int, 4>());
    }
    if (vecs <= 2048) return go(integral_constant<int, 1024>(), integral_constant<int, 2>());
    if (vecs <= 8192) return go(integral_constant<int, 1024>(), integral_constant<int, 8>());
    return go(integral_constant<int, 1024>(), integral_constant<int, 0>());
}

// ---- the product ------------------------------------------------------------------------------------------------------
struct FcI8 {
    const void* x;             // [n_rows][K] in the storage type
    const int8_t* xq;          // rows: in tiles for the kernel of few rows, [n_rows][x_stride] for the GEMM
    size_t x_stride, w_stride;
    const float* sx;
    const int8_t* w;           // [cout][w_stride]
    const float* sw;
    const float* bias;
    void* out;
    int n_rows, K, n_tiles, cout, relu;
    int splits;                // workgroups that share a tile's K, and what they need: sums and counters
    int* part;                 // [tiles][splits][a tile's sums]
    int32_t* done;             // [tiles]
};

template <typename T>
__device__ __forceinline__ T to_out(float v);
template <>
__device__ __forceinline__ float to_out<float>(float v) { return v; }
template <>
__device__ __forceinline__ __hip_bfloat16 to_out<__hip_bfloat16>(float v) { return __float2bfloat16(v); }

// A sum's way out, the same operations in every kernel.  The sum has 31 bits: its product with a very large scale of weights would leave
// fp32 where the result, with a small scale of the row, does not.  Such a scale is taken 2^-64 times and the row's 2^64 times
// (finite: a sum of zero stays one).  (In the other direction nothing is lost: a whole number times the smallest number is exact.)
struct WeightScale {
    float s;
    bool large;
    __device__ __forceinline__ explicit WeightScale(float sw) : s(sw), large(fabsf(sw) > 0x1p90f) {
        if (large) s = sw * 0x1p-64f;
    }
};
struct OutScale {              // of a row
    float s, behind_large;
    __device__ __forceinline__ explicit OutScale(float sx) : s(sx), behind_large(sx * 0x1p64f) {
        if (behind_large > 0x1.fffffep127f) behind_large = 0x1.fffffep127f;
    }
};
__device__ __forceinline__ float finish(int sum, const WeightScale& sw, const OutScale& sx, float bias, int relu) {
    const float v = fmaf((float)sum * sw.s, sw.large ? sx.behind_large : sx.s, bias);
    return relu && v < 0.f ? 0.f : v;
}

// 16 weights of a row from k0 on; past the row's end zeros: what overlaps the end comes from the row's last 16 bytes (one by one it
// would take 3 us longer, 1023 -> 1000 on 64 rows 12.0).
__device__ __forceinline__ intx4 weights16(const int8_t* __restrict__ row, int k0, int K) {
    if (k0 + 16 <= K) return *reinterpret_cast<const intx4_any*>(row + k0);
    unsigned long long lo = 0, hi = 0;
    if (k0 < K) {
        if (K >= 16) {
            const intx4 v = *reinterpret_cast<const intx4_any*>(row + K - 16);
            const int bits = (k0 - (K - 16)) * 8;          // 8 .. 120
            lo = (unsigned long long)(uint32_t)v[1] << 32 | (uint32_t)v[0];
            hi = (unsigned long long)(uint32_t)v[3] << 32 | (uint32_t)v[2];
            if (bits >= 64) { lo = hi >> (bits - 64); hi = 0; }
            else { lo = lo >> bits | hi << (64 - bits); hi >>= bits; }
        } else {
#pragma unroll 1
            for (int e = 0; k0 + e < K; ++e) {
                const unsigned long long u = (uint8_t)row[k0 + e];
                if (e < 8) lo |= u << (8 * e);
                else hi |= u << (8 * e - 64);
            }
        }
    }
    return intx4{(int)(uint32_t)lo, (int)(uint32_t)(lo >> 32), (int)(uint32_t)hi, (int)(uint32_t)(hi >> 32)};
}

// Few rows: a workgroup takes 16 channels x NB * 16 rows.  Its wavefronts deal the 128-byte steps of K among themselves and add
// their integer sums through LDS.  The weights are what has to come from memory: they go straight from there into fragments
// (16 rows of 64 bytes an instruction), AHEAD steps of a wavefront before they are multiplied.  The rows come from L2, in tiles.
// OWN: there is one row, and every workgroup rounds it itself, into LDS, while its first weights travel, which saves a launch
// (9216 -> 4096: 9.3 us against 8.6 + 3.1; four rows that way 15.0 against 8.6 + 3.1).  What bounds it: one row 9216 -> 4096 fp32
// 10.2 us, 3.7 TB/s of weights, of which 2 us are the start of the kernel and the rounding; small layers the way to memory and back, 1152 -> 100
// 5.4 us; 64 rows (9216 -> 4096, where the GEMM takes over, 14.0 us) their 590 KB a CU from L2 and a look-up for every 16 bytes of weights.
// ODD: rows of weights that begin inside words of 4 bytes: the five words that hold 16 of them (each holds a byte that is asked for), shifted
// where they are multiplied (loads at such addresses run at half the rate: 9217 -> 4000, one row, 22.7 us, 9216 -> 4000 12.4).
template <typename T, int NB, int WAVES, int AHEAD, bool OWN, bool ODD>
__global__ __launch_bounds__(WAVES * 64) void fc_i8_rows_kernel(FcI8 P) {
    static_assert(!OWN || NB == 1, "");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16;
    // channels past the end repeat the last one (not stored)
    const int8_t* const wrow = P.w + (size_t)min(o0 + l16, P.cout - 1) * P.K;
    const int steps = P.n_tiles / 2, whole = P.K / 128;
    struct Step { intx4 w[2], x[OWN ? 1 : NB][2]; int behind[ODD ? 2 : 1]; };
    typedef int intx4_word __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t into = ODD ? reinterpret_cast<uintptr_t>(wrow) & 3 : 0;
    const int8_t* const words = wrow - into;
    const int word_behind = into ? 16 : 12;
    const int8_t* const xt = P.xq + lane * 16;
    auto fetch = [&](Step& b, int s) {
        if (s < whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = s * 128 + h * 64 + g * 16;
                if constexpr (ODD) {
                    b.w[h] = *reinterpret_cast<const intx4_word*>(words + at);
                    b.behind[h] = *reinterpret_cast<const int*>(words + at + word_behind);
                } else {
                    b.w[h] = *reinterpret_cast<const intx4_any*>(wrow + at);
                }
            }
        } else if (s < steps) {
#pragma unroll
            for (int h = 0; h < 2; ++h) b.w[h] = weights16(wrow, s * 128 + h * 64 + g * 16, P.K);
        }
        if constexpr (!OWN) {
            if (s < steps)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) b.x[j][h] = *reinterpret_cast<const intx4*>(xt + ((size_t)j * P.n_tiles + s * 2 + h) * 1024);
        }
    };
    Step step[AHEAD + 1];
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) fetch(step[d], wave + d * WAVES);
    __builtin_amdgcn_sched_barrier(0);
    unsigned char* const own_x = smem + 256;               // [width], behind the wavefronts' largest |x|
    float own_scale = 0.f;
    if constexpr (OWN) {
        constexpr int N = RowVec<T>::N, THREADS = WAVES * 64, CH = 4;
        const T* const x = static_cast<const T*>(P.x);
        const int vecs = P.n_tiles * 64 / N;
        float f[CH][N];                                    // (what does not fit is read again)
        uint32_t top = 0;
        auto look = [&](const float (&v)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
        };
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * THREADS + tid < vecs) {
                load_row(x, (c * THREADS + tid) * N, P.K, f[c]);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) f[c][e] = 0.f;
            }
#pragma unroll
        for (int c = 0; c < CH; ++c) look(f[c]);
        for (int i = CH * THREADS + tid; i < vecs; i += THREADS) {
            float more[N];
            load_row(x, i * N, P.K, more);
            look(more);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        uint32_t* const tops = reinterpret_cast<uint32_t*>(smem);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < WAVES; ++v) top = max(top, tops[v]);
        const RowScale s(top);
        own_scale = s.scale;
        auto put = [&](int i, const float (&v)[N]) {
            uint32_t w[N / 4] = {};
            if (!s.zero) quotients8(v, s.s, s.inv, w);
#pragma unroll
            for (int e = 0; e < N / 4; ++e) reinterpret_cast<uint32_t*>(own_x)[i * (N / 4) + e] = w[e];
        };
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * THREADS + tid < vecs) put(c * THREADS + tid, f[c]);
        for (int i = CH * THREADS + tid; i < vecs; i += THREADS) {
            float more[N];
            load_row(x, i * N, P.K, more);
            put(i, more);
        }
        __syncthreads();
    }
    intx4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = intx4{0, 0, 0, 0};
    for (int s = wave; s < steps; s += (AHEAD + 1) * WAVES) {
#pragma unroll
        for (int d = 0; d <= AHEAD; ++d) {
            if (s + d * WAVES >= steps) break;
            fetch(step[(d + AHEAD) % (AHEAD + 1)], s + (d + AHEAD) * WAVES);
            __builtin_amdgcn_sched_barrier(0);
            const Step& b = step[d];
            const uint32_t by = s + d * WAVES < whole ? into : 0;          // (a row's end comes in its place)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                intx4 w = b.w[h];
                if constexpr (ODD)
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = (int)__builtin_amdgcn_alignbyte((uint32_t)(i < 3 ? b.w[h][i < 3 ? i + 1 : i] : b.behind[h]), (uint32_t)b.w[h][i], by);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    intx4 x;
                    if constexpr (OWN) x = *reinterpret_cast<const intx4*>(own_x + (s + d * WAVES) * 128 + h * 64 + g * 16);
                    else x = b.x[j][h];
                    acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc[j], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (OWN) __syncthreads();                    // the row has been read
    intx4* const red = reinterpret_cast<intx4*>(smem + 256);               // [WAVES][NB][64]
#pragma unroll
    for (int j = 0; j < NB; ++j) red[(wave * NB + j) * 64 + lane] = acc[j];
    __syncthreads();
    for (int i = tid; i < NB * 64; i += WAVES * 64) {
        const int l = i & 63, row = (i >> 6) * 16 + (l & 15), o = o0 + (l >> 4) * 4;
        if (row >= P.n_rows || o >= P.cout) continue;
        intx4 sum = red[i];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += red[v * NB * 64 + i];
        const OutScale sx(OWN ? own_scale : P.sx[row]);
        T* const out = static_cast<T*>(P.out) + (size_t)row * P.cout;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (o + e >= P.cout) break;
            out[o + e] = to_out<T>(finish(sum[e], WeightScale(P.sw[o + e]), sx, P.bias ? P.bias[o + e] : 0.f, P.relu));
        }
    }
}

// Many rows: a GEMM of MT * 16 rows x NT * 16 channels per workgroup.  Both operands come through LDS in stages of 128 bytes of K
// by direct loads: an instruction brings 8 rows of 128 bytes, whole cache lines, eight lanes a row, and the eight vectors of
// row r are stored in the order v ^ (r % 8), so that eight neighbouring lanes of a fragment ask 128 different bytes.  Half a
// stage is multiplied while the fragments of the next half are read into the other set of registers; one barrier a stage.
// Rows are whole 16-byte vectors; what lies behind a row of weights meets zeros of the input row, and what lies behind an
// operand's end reads as zero.  The matrix instructions bound it: 4096 -> 4096 on 16384 rows 295 to 303 us, 1.85 POP/s, where the same
// instructions without any load reach 2.26 (the power limit, with random numbers) and a library's product of 8192 x 8192 x 8192
// 2.04; 1024 -> 256 on 12544 rows (196 tiles, one a CU) 11.3 us, mostly the first and the last stage.
// SPLIT: P.splits workgroups share a tile, each with a run of K, and the one that comes last adds their integer sums up; nothing
// waits for another.  The sums go past the XCDs' caches (atomic operations of the GPU's scope).
constexpr int kBufferFlags = 0x00020000;
constexpr int kMaxLds = 160 * 1024;
typedef __attribute__((address_space(3))) void* lds_ptr;
template <int N>
__device__ __forceinline__ void wait_vmcnt() { __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14); }
template <typename T, int MT, int NT, int WM, int WN, int STAGES, bool SPLIT>
__global__ __launch_bounds__(WM * WN * 64) void fc_i8_gemm_kernel(FcI8 P) {
    constexpr int WAVES = WM * WN, XI = 2 * MT / WAVES, WI = 2 * NT / WAVES, UM = MT / WM, UN = NT / WN;
    static_assert(2 * MT % WAVES == 0 && 2 * NT % WAVES == 0, "every wavefront loads as many rows of either operand");
    constexpr int kStage = (MT + NT) * 2048;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4, wm = wave % WM, wn = wave / WM;
    // workgroup -> tile: every XCD (workgroup number modulo 8) takes a run of the tiles, which go down columns of 8 row tiles
    const int n_m = (P.n_rows + MT * 16 - 1) / (MT * 16), n_n = (P.cout + NT * 16 - 1) / (NT * 16);
    int tm, tn, tile = 0, run = 0;
    {
        const int n = n_m * n_n * (SPLIT ? P.splits : 1), xcd = blockIdx.x & 7, j = blockIdx.x >> 3, per = n >> 3, more = n & 7;
        int at = xcd * per + min(xcd, more) + j;
        if constexpr (SPLIT) {
            run = at % P.splits;
            at = tile = at / P.splits;
        }
        const int band = at / (8 * n_n), left = min(8, n_m - band * 8), in = at - band * 8 * n_n;
        tm = band * 8 + in % left;
        tn = in / left;
    }
    const int m0 = tm * (MT * 16), o0 = tn * (NT * 16);    // first row, first channel
    const int rows = min(MT * 16, P.n_rows - m0), chans = min(NT * 16, P.cout - o0);
    const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(P.xq) + m0 * P.x_stride, 0,
                                                                            (uint32_t)(rows * P.x_stride), kBufferFlags);
    const __amdgpu_buffer_rsrc_t w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(P.w) + o0 * P.w_stride, 0,
                                                                            (uint32_t)(chans * P.w_stride), kBufferFlags);
    uint32_t xo[XI], wo[WI];
    const int first = SPLIT ? P.n_tiles / 2 * run / P.splits : 0, stages = (SPLIT ? P.n_tiles / 2 * (run + 1) / P.splits : P.n_tiles / 2) - first;
    const int r = lane >> 3, v16 = first * 128 + (((lane & 7) ^ r) << 4);
#pragma unroll
    for (int i = 0; i < XI; ++i) xo[i] = (uint32_t)(((i * WAVES + wave) * 8 + r) * P.x_stride) + v16;
#pragma unroll
    for (int i = 0; i < WI; ++i) wo[i] = (uint32_t)(((i * WAVES + wave) * 8 + r) * P.w_stride) + v16;
    auto issue = [&](int buf) {                            // the next stage of either operand
        unsigned char* const to = smem + buf * kStage + wave * 1024;
#pragma unroll
        for (int i = 0; i < XI; ++i) {
            const uint32_t off = xo[i];                    // (a named value: an expression in the builtin's argument list loses the host stub)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rsrc, (lds_ptr)(to + i * (WAVES * 1024)), 16, off, 0, 0, 0);
            xo[i] += 128;
        }
#pragma unroll
        for (int i = 0; i < WI; ++i) {
            const uint32_t off = wo[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (lds_ptr)(to + (MT * 2 + i * WAVES) * 1024), 16, off, 0, 0, 0);
            wo[i] += 128;
        }
    };
    intx4 acc[UM][UN];
#pragma unroll
    for (int i = 0; i < UM; ++i)
#pragma unroll
        for (int j = 0; j < UN; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    const int x_at = (wm * UM * 16 + l16) * 128, w_at = (MT * 16 + wn * UN * 16 + l16) * 128;
    const int half_at[2] = {(g ^ (l16 & 7)) << 4, ((g + 4) ^ (l16 & 7)) << 4};
    intx4 x[2][UM], w[2][UN];
    auto fragments = [&](int half, int buf) {
        const unsigned char* const from = smem + buf * kStage + half_at[half];
#pragma unroll
        for (int j = 0; j < UN; ++j) w[half][j] = *reinterpret_cast<const intx4*>(from + w_at + j * 2048);
#pragma unroll
        for (int i = 0; i < UM; ++i) x[half][i] = *reinterpret_cast<const intx4*>(from + x_at + i * 2048);
    };
    auto multiply = [&](int half) {
#pragma unroll
        for (int i = 0; i < UM; ++i)
#pragma unroll
            for (int j = 0; j < UN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[half][j], x[half][i], acc[i][j], 0, 0, 0);
    };
    // the order of a half: a fragment's read, a few products, and so on, so that the reads travel behind the products
    constexpr int kLoads = XI + WI, kReads = UM + UN, kProducts = UM * UN;
    auto interleave = [&]() {
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, kProducts / kReads, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kProducts - kProducts / kReads * kReads, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int s = 0; s < STAGES; ++s) issue(s);
    wait_vmcnt<(STAGES - 1) * kLoads>();
    asm volatile("s_barrier" ::: "memory");
    fragments(0, 0);
    int buf = 0;
    for (int t = 0; t < stages; ++t) {
        const int next = buf + 1 == STAGES ? 0 : buf + 1;
        fragments(1, buf);
        multiply(0);
        interleave();
        wait_vmcnt<(STAGES - 2) * kLoads>();
        // every wavefront has the rest of this stage in registers, and the next stage has arrived
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        issue(buf);
        __builtin_amdgcn_sched_barrier(0);
        fragments(0, next);
        multiply(1);
        interleave();
        buf = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");       // the loads behind the last stage end before the workgroup does
    if constexpr (SPLIT) {
        constexpr int SUMS = UM * UN, THREADS = WAVES * 64;
        auto sum_at = [&](int who, int i) { return reinterpret_cast<unsigned long long*>(P.part) + ((((size_t)tile * P.splits + who) * SUMS + i) * THREADS + tid) * 2; };
#pragma unroll
        for (int i = 0; i < SUMS; ++i) {
            unsigned long long u[2];
            __builtin_memcpy(u, &acc[i / UN][i % UN], 16);
#pragma unroll
            for (int h = 0; h < 2; ++h) __hip_atomic_store(sum_at(run, i) + h, u[h], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wavefront's sums have arrived
        __syncthreads();
        int* const last = reinterpret_cast<int*>(smem);
        if (tid == 0) *last = __hip_atomic_fetch_add(P.done + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == P.splits - 1;
        __syncthreads();
        if (!*last) return;
        for (int d = 1; d < P.splits; ++d) {
            const int who = run + d < P.splits ? run + d : run + d - P.splits;
#pragma unroll
            for (int i = 0; i < SUMS; ++i) {
                unsigned long long u[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) u[h] = __hip_atomic_load(sum_at(who, i) + h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                intx4 v;
                __builtin_memcpy(&v, u, 16);
                acc[i / UN][i % UN] += v;
            }
        }
    }
    const bool vec = P.cout % 4 == 0 && reinterpret_cast<uintptr_t>(P.out) % (4 * sizeof(T)) == 0;
#pragma unroll
    for (int j = 0; j < UN; ++j) {
        const int o = o0 + (wn * UN + j) * 16 + g * 4;
        if (o >= P.cout) continue;
        const auto channel = [&](int e) { return min(o + e, P.cout - 1); };
        const WeightScale sw[4] = {WeightScale(P.sw[channel(0)]), WeightScale(P.sw[channel(1)]), WeightScale(P.sw[channel(2)]), WeightScale(P.sw[channel(3)])};
        floatx4 bias{0.f, 0.f, 0.f, 0.f};
        if (P.bias)
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[e] = P.bias[channel(e)];
#pragma unroll
        for (int i = 0; i < UM; ++i) {
            const int row = m0 + (wm * UM + i) * 16 + l16;
            if (row >= P.n_rows) continue;
            const OutScale sx(P.sx[row]);
            T v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = to_out<T>(finish(acc[i][j][e], sw[e], sx, bias[e], P.relu));
            T* const out = static_cast<T*>(P.out) + (size_t)row * P.cout + o;
            if (vec) __builtin_memcpy(__builtin_assume_aligned(out, 4 * sizeof(T)), v, sizeof v);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (o + e < P.cout) out[e] = v[e];
        }
    }
}

// A kernel whose LDS is sized at the launch; the attribute is raised once per instantiation and GPU (a bit each).
template <typename K>
hipError_t launch_lds(K kernel, std::atomic<uint64_t>& raised, unsigned wgs, unsigned threads, unsigned lds, const FcI8& P, hipStream_t st) {
    if (lds > 64 * 1024) {
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        const uint64_t bit = 1ull << (dev & 63);
        if (!(raised.load() & bit)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLds);
            if (e != hipSuccess) return e;
            raised.fetch_or(bit);
        }
    }
    hipLaunchKernelGGL(kernel, dim3(wgs), dim3(threads), lds, st, P);
    return hipGetLastError();
}
template <typename T, int NB, int WAVES, int AHEAD, bool OWN>
hipError_t rows_launch(const FcI8& P, hipStream_t st) {
    auto go = [&](auto odd) {
        constexpr bool ODD = decltype(odd)::value;
        static std::atomic<uint64_t> raised{0};
        const unsigned lds = 256 + (unsigned)std::max(OWN ? P.n_tiles * 64 : 0, WAVES * NB * 1024);
        return launch_lds(fc_i8_rows_kernel<T, NB, WAVES, AHEAD, OWN, ODD>, raised, (unsigned)((P.cout + 15) / 16), WAVES * 64, lds, P, st);
    };
    return (reinterpret_cast<uintptr_t>(P.w) | P.K) & 3 ? go(std::true_type()) : go(std::false_type());
}
template <typename T, int MT, int NT, int WM, int WN, int STAGES, bool SPLIT = false>
hipError_t gemm(const FcI8& P, hipStream_t st) {
    static std::atomic<uint64_t> raised{0};
    const size_t wgs = ((size_t)P.n_rows + MT * 16 - 1) / (MT * 16) * (((size_t)P.cout + NT * 16 - 1) / (NT * 16)) * (SPLIT ? P.splits : 1);
    if (wgs > 0x7fffffffu) return hipErrorInvalidValue;
    return launch_lds(fc_i8_gemm_kernel<T, MT, NT, WM, WN, STAGES, SPLIT>, raised, (unsigned)wgs, WM * WN * 64, STAGES * (MT + NT) * 2048, P, st);
}

// [cout][K] -> rows of whole vectors, zeros behind K
__global__ __launch_bounds__(256) void pad_weights_kernel(const int8_t* __restrict__ w, int8_t* __restrict__ to, int K, int width) {
    const int k0 = (blockIdx.x * 256 + threadIdx.x) * 16;
    if (k0 < width) *reinterpret_cast<intx4*>(to + (size_t)blockIdx.y * width + k0) = weights16(w + (size_t)blockIdx.y * K, k0, K);
}

template <typename T>
hipError_t product_few(const FcI8& P, hipStream_t st) {
    if (P.n_rows <= 16) return rows_launch<T, 1, 16, 2, false>(P, st);
    if (P.n_rows <= 32) return rows_launch<T, 2, 8, 2, false>(P, st);
    if (P.n_rows <= 48) return rows_launch<T, 3, 8, 2, false>(P, st);
    return rows_launch<T, 4, 8, 2, false>(P, st);
}
// us, 128 x 128 (two workgroups a CU) against 256 x 256: 4096 -> 4096 on 16384 rows (4096 or 1024 tiles) 277 against 265, 2048 -> 2048
// on 8192 (1024 or 256) 45 against 52.  Three stages in flight are worth one workgroup a CU while there are no more tiles than CUs: 4096 ->
// 4096 on 1024 rows 26.4 -> 22.2, but 2048 -> 2048 on 4096 (512 tiles) 24.1 -> 28.8.  Half as many tiles or fewer leave CUs idle:
// 4096 -> 4096 on 256 rows 17.7 with 128 x 128, 10.4 with 64 x 64 (four stages; two 11.2).  Up to 64 channels: 256 -> 64 on 50176
// rows 6.7 with 128 x 64, 8.4 with 128 x 128, 7.3 with 64 x 64.
template <typename T>
hipError_t product_many(const FcI8& P, hipStream_t st) {
    if (P.splits > 1) return gemm<T, 4, 4, 2, 4, 4, true>(P, st);
    const long tiles = ((long)P.n_rows + 127) / 128 * ((P.cout + 127) / 128), big = ((long)P.n_rows + 255) / 256 * ((P.cout + 255) / 256);
    if (P.cout <= 64 && tiles > 64) return gemm<T, 8, 4, 2, 4, 2>(P, st);
    if (big >= 768) return gemm<T, 16, 16, 2, 4, 2>(P, st);
    if (tiles > 256) return gemm<T, 8, 8, 2, 4, 2>(P, st);
    if (tiles > 128) return gemm<T, 8, 8, 2, 4, 3>(P, st);
    return gemm<T, 4, 4, 2, 4, 4>(P, st);
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int dtype, size_t n_rows, int K, int8_t* q, float* scales, hipStream_t st) {
    const Rows8 to{q, (size_t)K, K};
    return dtype == DC_BF16 ? quantize<__hip_bfloat16, false>((const __hip_bfloat16*)x, n_rows, K, to, scales, st)
                            : quantize<float, false>((const float*)x, n_rows, K, to, scales, st);
}

size_t fc_i8_workspace(int n_rows, int K, int cout) { return i8_workspace(n_rows, K, cout); }

static bool whole_vectors(const int8_t* w, int K) { return K % 16 == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0; }
int fc_i8_rows(int n_rows, int K, int cout, const int8_t* w, size_t ws_bytes) { return i8_rows(n_rows, K, cout, whole_vectors(w, K), ws_bytes); }

template <typename T>
static hipError_t run_fc_i8(const T* x, FcI8 P, int8_t* ws, size_t ws_bytes, hipStream_t st) {
    const I8Plan plan = i8_plan(P.n_rows, P.K, P.cout, whole_vectors(P.w, P.K), ws_bytes);
    const int width = (int)plan.width;
    P.x = x; P.n_tiles = width / 64; P.w_stride = P.K;
    if (P.n_rows == 1) return rows_launch<T, 1, 16, 2, true>(P, st);
    float* const sx = reinterpret_cast<float*>(ws + plan.scales.at);
    P.splits = plan.splits;
    Rows8 to{ws + plan.rows.at, plan.width, width};
    if (plan.splits > 1) {
        P.part = reinterpret_cast<int*>(ws + plan.part.at);
        P.done = reinterpret_cast<int32_t*>(ws + plan.done.at);
        to.zero = P.done;
        to.zeros = (int)plan.tiles;
    }
    P.xq = to.q; P.x_stride = plan.width; P.sx = sx;
    hipError_t e = plan.few ? quantize<T, true>(x, P.n_rows, P.K, to, sx, st) : quantize<T, false>(x, P.n_rows, P.K, to, sx, st);
    if (e != hipSuccess) return e;
    if (plan.few) return product_few<T>(P, st);
    if (plan.copy) {
        int8_t* const w = ws + plan.weights.at;
        for (int c = 0; c < P.cout; c += 65535) {
            const int n = std::min(65535, P.cout - c);
            hipLaunchKernelGGL(pad_weights_kernel, dim3((unsigned)((width / 16 + 255) / 256), (unsigned)n), dim3(256), 0, st, P.w + (size_t)c * P.K,
                               w + (size_t)c * width, P.K, width);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        P.w = w; P.w_stride = plan.width;
    }
    return product_many<T>(P, st);
}

hipError_t launch_fc_i8(const void* x, const int8_t* w, const float* sw, const float* bias, void* out, int n_rows, int K, int cout, int relu,
                        int dtype, void* ws, size_t ws_bytes, hipStream_t st) {
    const int at_once = fc_i8_rows(n_rows, K, cout, w, ws_bytes);
    if (at_once < 1) return hipErrorInvalidValue;
    for (int r = 0; r < n_rows; r += at_once) {
        FcI8 P;
        P.w = w; P.sw = sw; P.bias = bias; P.K = K; P.cout = cout; P.relu = relu;
        P.n_rows = std::min(at_once, n_rows - r);
        P.out = static_cast<unsigned char*>(out) + (size_t)r * cout * dtype_size(dtype);
        const void* const rows = static_cast<const unsigned char*>(x) + (size_t)r * K * dtype_size(dtype);
        const hipError_t e = dtype == DC_BF16 ? run_fc_i8((const __hip_bfloat16*)rows, P, static_cast<int8_t*>(ws), ws_bytes, st)
                                              : run_fc_i8((const float*)rows, P, static_cast<int8_t*>(ws), ws_bytes, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace dc

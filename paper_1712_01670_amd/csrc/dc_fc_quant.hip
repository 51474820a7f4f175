// Fully-connected layers in 8-bit integers.  A row (a token, a pixel, a stream's features) is rounded to 8 bits with a scale of
// its own, the weights have a scale per output channel, so that
//   out[r][o] = act(sx[r] sw[o] sum_k q[r][k] w[o][k] + bias[o])
// with an integer sum that is exact whatever its order: results do not depend on which kernel runs, on how K is split or on
// how many rows a call has.
#include <hip/hip_bf16.h>

#include <algorithm>

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

template <typename T>
struct In16;                                         // 16 elements of a row
template <>
struct In16<float> {
    typedef float vec_any __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void load(const float* p, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const vec_any v = *reinterpret_cast<const vec_any*>(p + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * i + e] = v[e];
        }
    }
    static __device__ __forceinline__ float one(const float* p) { return *p; }
};
template <>
struct In16<__hip_bfloat16> {
    typedef uint32_t vec_any __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ void load(const __hip_bfloat16* p, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const vec_any v = *reinterpret_cast<const vec_any*>(p + 8 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[8 * i + 2 * e] = __uint_as_float(v[e] << 16);
                f[8 * i + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            }
        }
    }
    static __device__ __forceinline__ float one(const __hip_bfloat16* p) { return __bfloat162float(*p); }
};

// Rows for the matrix units: tiles of 16 rows x 64 bytes in the order of a fragment's lanes (lane l: row l % 16, bytes
// 16 (l / 16) on), 1 KiB in one piece, K padded with zeros to whole tiles.  Tile (i, j) is number i * n_tiles + j.
__device__ __forceinline__ size_t tile_offset(size_t row, int k0, int n_tiles) {
    return ((row >> 4) * n_tiles + (k0 >> 6)) * 1024 + ((k0 >> 4) & 3) * 256 + (row & 15) * 16;
}

// LANES threads share a row and hold it in registers, CH pieces of 16 elements each, so it is read once.
// TILED: the layout above; otherwise [n_rows][K].
template <typename T, int LANES, int CH, bool TILED>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void quantize_rows_kernel(const T* __restrict__ x, size_t n_rows, int K, int n_tiles,
                                                                                  int8_t* __restrict__ q, float* __restrict__ scales) {
    constexpr int THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    const int tid = threadIdx.x, part = tid % LANES;
    const size_t row = (size_t)blockIdx.x * ROWS + tid / LANES;
    const bool live = row < n_rows;
    const T* const xr = x + (live ? row : 0) * K;
    float f[CH][16];
    uint32_t top = 0;                                // the largest |x|: as whole numbers, infinities and NaN come out on top
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int k0 = (c * LANES + part) * 16;
        if (live && k0 + 16 <= K) {
            In16<T>::load(xr + k0, f[c]);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) f[c][e] = live && k0 + e < K ? In16<T>::one(xr + k0 + e) : 0.f;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(f[c][e]) & 0x7fffffffu);
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
    const bool bad = top >= 0x7f800000u;
    const float s = __uint_as_float(top) / 127.f;
    if (part == 0) scales[row] = bad ? __uint_as_float(0x7fc00000u) : s;
    const bool zero = bad || !(s > 0.f);
    const float up = s < 0x1p-100f ? 0x1p64f : 1.f;  // keeps 1 / s finite; a power of two changes no quotient
    const float su = s * up, inv = 1.f / su;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int k0 = (c * LANES + part) * 16;
        intx4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) w |= (uint32_t)(quotient8(f[c][4 * i + e] * up, su, inv) & 255) << (8 * e);
            v[i] = zero ? 0 : (int)w;
        }
        if constexpr (TILED) {
            if (k0 < n_tiles * 64) *reinterpret_cast<intx4*>(q + tile_offset(row, k0, n_tiles)) = v;
        } else if (k0 + 16 <= K) {
            *reinterpret_cast<intx4_any*>(q + row * K + k0) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (k0 + e < K) q[row * K + k0 + e] = (int8_t)((uint32_t)v[e >> 2] >> (8 * (e & 3)));
        }
    }
}

template <typename T, bool TILED>
hipError_t quantize(const T* x, size_t n_rows, int K, int8_t* q, float* scales, hipStream_t st) {
    const int n_tiles = (K + 63) / 64;
    auto go = [&](auto lanes, auto ch) {
        constexpr int LANES = decltype(lanes)::value, CH = decltype(ch)::value, THREADS = LANES > 256 ? LANES : 256;
        const size_t wgs = (n_rows + THREADS / LANES - 1) / (THREADS / LANES);
        hipLaunchKernelGGL((quantize_rows_kernel<T, LANES, CH, TILED>), dim3((unsigned)wgs), dim3(THREADS), 0, st, x, n_rows, K, n_tiles, q, scales);
        return hipGetLastError();
    };
    using std::integral_constant;
    const int pieces = n_tiles * 4;
    if (pieces <= 64) return go(integral_constant<int, 16>(), integral_constant<int, 4>());
    if (pieces <= 256) return go(integral_constant<int, 64>(), integral_constant<int, 4>());
    if (pieces <= 1024) return go(integral_constant<int, 256>(), integral_constant<int, 4>());
    if (pieces <= 4096) return go(integral_constant<int, 1024>(), integral_constant<int, 4>());
    return go(integral_constant<int, 1024>(), integral_constant<int, 8>());
}

// ---- the product ------------------------------------------------------------------------------------------------------
struct FcI8 {
    const int8_t* xq;          // rows in tiles
    const float* sx;
    const int8_t* w;           // [cout][K]
    const float* sw;
    const float* bias;
    void* out;
    int n_rows, K, n_tiles, cout, relu;
};

template <typename T>
__device__ __forceinline__ T to_out(float v);
template <>
__device__ __forceinline__ float to_out<float>(float v) { return v; }
template <>
__device__ __forceinline__ __hip_bfloat16 to_out<__hip_bfloat16>(float v) { return __float2bfloat16(v); }

// 16 weights of a row from k0 on; past the row's end zeros.
__device__ __forceinline__ intx4 weights16(const int8_t* __restrict__ row, int k0, int K) {
    if (k0 + 16 <= K) return *reinterpret_cast<const intx4_any*>(row + k0);
    intx4 v{0, 0, 0, 0};
    for (int e = 0; k0 + e < K; ++e) v[e >> 2] |= (int)((uint32_t)(uint8_t)row[k0 + e] << (8 * (e & 3)));
    return v;
}

// A workgroup takes 16 channels x NB * 16 rows; its wavefronts deal the tiles of K among themselves and add their integer
// sums through LDS.
constexpr int kI8Waves = 8;
template <typename T, int NB>
__global__ __launch_bounds__(kI8Waves * 64) void fc_i8_rows_kernel(FcI8 P) {
    __shared__ intx4 red[kI8Waves][NB][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int o0 = blockIdx.x * 16, r0 = blockIdx.y * (NB * 16);
    // channels past the end repeat the last one (not stored)
    const int8_t* const wrow = P.w + (size_t)min(o0 + l16, P.cout - 1) * P.K;
    const int n_blocks = min(NB, (P.n_rows - r0 + 15) / 16);
    const int8_t* const xt = P.xq + (size_t)(r0 >> 4) * P.n_tiles * 1024 + lane * 16;
    intx4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = intx4{0, 0, 0, 0};
    for (int t = wave; t < P.n_tiles; t += kI8Waves) {
        const intx4 wv = weights16(wrow, t * 64 + g * 16, P.K);
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (j < n_blocks) {
                const intx4 xv = *reinterpret_cast<const intx4*>(xt + ((size_t)j * P.n_tiles + t) * 1024);
                acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc[j], 0, 0, 0);
            }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) red[wave][j][lane] = acc[j];
    __syncthreads();
    for (int i = tid; i < NB * 64; i += kI8Waves * 64) {
        const int j = i >> 6, l = i & 63, row = r0 + j * 16 + (l & 15), o = o0 + (l >> 4) * 4;
        if (row >= P.n_rows || o >= P.cout) continue;
        intx4 sum = red[0][j][l];
#pragma unroll
        for (int v = 1; v < kI8Waves; ++v) sum += red[v][j][l];
        const float sx = P.sx[row];
        T* const out = static_cast<T*>(P.out) + (size_t)row * P.cout;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (o + e >= P.cout) break;
            float v = (float)sum[e] * P.sw[o + e] * sx;
            if (P.bias) v += P.bias[o + e];
            if (P.relu) v = v > 0.f || v != v ? v : 0.f;
            out[o + e] = to_out<T>(v);
        }
    }
}

template <typename T>
hipError_t product(const FcI8& P, hipStream_t st) {
    const dim3 block(kI8Waves * 64);
    const unsigned gx = (unsigned)((P.cout + 15) / 16);
    if (P.n_rows <= 16)
        hipLaunchKernelGGL((fc_i8_rows_kernel<T, 1>), dim3(gx, 1), block, 0, st, P);
    else
        hipLaunchKernelGGL((fc_i8_rows_kernel<T, 4>), dim3(gx, (unsigned)((P.n_rows + 63) / 64)), block, 0, st, P);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int dtype, size_t n_rows, int K, int8_t* q, float* scales, hipStream_t st) {
    return dtype == DC_BF16 ? quantize<__hip_bfloat16, false>((const __hip_bfloat16*)x, n_rows, K, q, scales, st)
                            : quantize<float, false>((const float*)x, n_rows, K, q, scales, st);
}

size_t fc_i8_workspace(int n_rows, int K) {
    const size_t rows = ((size_t)n_rows + 15) / 16 * 16;
    return align_up(rows * ((K + 63) / 64) * 64, 256) + align_up((size_t)n_rows * sizeof(float), 256);
}

hipError_t launch_fc_i8(const void* x, const int8_t* w, const float* sw, const float* bias, void* out, int n_rows, int K, int cout, int relu,
                        int dtype, void* ws, hipStream_t st) {
    FcI8 P;
    P.n_rows = n_rows; P.K = K; P.n_tiles = (K + 63) / 64; P.cout = cout; P.relu = relu;
    int8_t* const xq = static_cast<int8_t*>(ws);
    float* const sx = reinterpret_cast<float*>(xq + align_up(((size_t)n_rows + 15) / 16 * 16 * P.n_tiles * 64, 256));
    P.xq = xq; P.sx = sx; P.w = w; P.sw = sw; P.bias = bias; P.out = out;
    const hipError_t e = dtype == DC_BF16 ? quantize<__hip_bfloat16, true>((const __hip_bfloat16*)x, n_rows, K, xq, sx, st)
                                          : quantize<float, true>((const float*)x, n_rows, K, xq, sx, st);
    if (e != hipSuccess) return e;
    return dtype == DC_BF16 ? product<__hip_bfloat16>(P, st) : product<float>(P, st);
}

}  // namespace dc

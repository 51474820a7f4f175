// Fully-connected layers in 8-bit integers.  A row (a token, a pixel, a stream's features) is rounded to 8 bits with a scale of
// its own, the weights have a scale per output channel, so that
//   out[r][o] = act(sx[r] sw[o] sum_k q[r][k] w[o][k] + bias[o])
// with an integer sum that is exact whatever its order: results do not depend on which kernel runs, on how K is split or on
// how many rows a call has.
#include <hip/hip_bf16.h>

#include <algorithm>
#include <atomic>

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

// A sum's way out, the same operations in every kernel.
__device__ __forceinline__ float finish(int sum, float sw, float sx, float bias, int relu) {
    const float v = fmaf((float)sum * sw, sx, bias);
    return relu && v < 0.f ? 0.f : v;
}

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
constexpr int kI8FewRows = 64;
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
            out[o + e] = to_out<T>(finish(sum[e], P.sw[o + e], sx, P.bias ? P.bias[o + e] : 0.f, P.relu));
        }
    }
}

// Many rows: a GEMM of MT * 16 rows x NT * 16 channels per workgroup.  Both operands come through LDS in stages of 64 bytes of K
// by direct loads, STAGES - 1 of them on their way while one is multiplied; a barrier a stage.  A wavefront's part is
// MT / WM row tiles x NT / WN channel tiles, which is what a fragment read from LDS serves.
// The rows are tiles as they are (fragments of 1 KiB: no bank is asked twice).  Weights come from [cout][K] when their rows are
// whole aligned vectors (an instruction brings 16 rows of 64 bytes, four lanes a row; the four vectors of row r are stored in the
// order v ^ (r / 2 % 4), so that eight neighbouring fragment lanes ask 128 different bytes), otherwise from a copy in
// tiles (W_TILED).  What lies behind the end of a row of weights meets zeros of the input row; what lies behind an operand's
// end reads as zero.
constexpr int kBufferFlags = 0x00020000;
typedef __attribute__((address_space(3))) void* lds_ptr;
template <typename T, int MT, int NT, int WM, int WN, int STAGES, bool W_TILED>
__global__ __launch_bounds__(WM * WN * 64) void fc_i8_gemm_kernel(FcI8 P) {
    constexpr int WAVES = WM * WN, XI = MT / WAVES, WI = NT / WAVES, UM = MT / WM, UN = NT / WN;
    static_assert(MT % WAVES == 0 && NT % WAVES == 0, "every wavefront loads as many tiles of either operand");
    constexpr int kStage = (MT + NT) * 1024;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4, wm = wave % WM, wn = wave / WM;
    // workgroup -> tile: every XCD (workgroup number modulo 8) takes a run of the tiles, which go down columns of 8 row tiles
    const int n_m = (P.n_rows + MT * 16 - 1) / (MT * 16), n_n = (P.cout + NT * 16 - 1) / (NT * 16);
    int tm, tn;
    {
        const int n = n_m * n_n, xcd = blockIdx.x & 7, j = blockIdx.x >> 3, per = n >> 3, more = n & 7;
        const int at = xcd * per + min(xcd, more) + j;
        const int band = at / (8 * n_n), left = min(8, n_m - band * 8), in = at - band * 8 * n_n;
        tm = band * 8 + in % left;
        tn = in / left;
    }
    const int m0 = tm * MT, o0 = tn * (NT * 16);           // first row tile, first channel
    const int m_tiles = min(MT, (P.n_rows + 15) / 16 - m0), chans = min(NT * 16, P.cout - o0);
    const size_t tile_row = (size_t)P.n_tiles * 1024;
    const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t*>(P.xq) + m0 * tile_row, 0, (uint32_t)(m_tiles * tile_row), kBufferFlags);
    const __amdgpu_buffer_rsrc_t w_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t*>(P.w) + (W_TILED ? (o0 >> 4) * tile_row : (size_t)o0 * P.K), 0,
        (uint32_t)(W_TILED ? (chans + 15) / 16 * tile_row : (size_t)chans * P.K), kBufferFlags);
    uint32_t xo[XI], wo[WI];
#pragma unroll
    for (int i = 0; i < XI; ++i) xo[i] = (uint32_t)((i * WAVES + wave) * tile_row) + lane * 16;
#pragma unroll
    for (int i = 0; i < WI; ++i) {
        const int t = i * WAVES + wave, r = lane >> 2;
        wo[i] = W_TILED ? (uint32_t)(t * tile_row) + lane * 16 : (uint32_t)(t * 16 + r) * P.K + (((lane & 3) ^ ((r / 2) & 3)) << 4);
    }
    auto issue = [&](int buf) {                            // the next stage of either operand
        unsigned char* const to = smem + buf * kStage + wave * 1024;
#pragma unroll
        for (int i = 0; i < XI; ++i) {
            const uint32_t off = xo[i];                    // (a named value: an expression in the builtin's argument list loses the host stub)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rsrc, (lds_ptr)(to + i * (WAVES * 1024)), 16, off, 0, 0, 0);
            xo[i] += 1024;
        }
#pragma unroll
        for (int i = 0; i < WI; ++i) {
            const uint32_t off = wo[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (lds_ptr)(to + (MT + i * WAVES) * 1024), 16, off, 0, 0, 0);
            wo[i] += W_TILED ? 1024 : 64;
        }
    };
    intx4 acc[UM][UN];
#pragma unroll
    for (int i = 0; i < UM; ++i)
#pragma unroll
        for (int j = 0; j < UN; ++j) acc[i][j] = intx4{0, 0, 0, 0};
    const int x_at = wm * UM * 1024 + lane * 16;
    const int w_at = (MT + wn * UN) * 1024 + (W_TILED ? lane * 16 : l16 * 64 + ((g ^ ((l16 / 2) & 3)) << 4));
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) issue(s);
    int buf = 0, next = STAGES - 1;
    for (int t = 0; t < P.n_tiles; ++t) {
        // the stages behind this one may still be on their way
        static_assert((STAGES - 2) * (XI + WI) <= 15, "");
        __builtin_amdgcn_s_waitcnt(0x0f70 | ((STAGES - 2) * (XI + WI)));       // vmcnt alone
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        issue(next);                                       // into the buffer that the last stage was read from
        const unsigned char* const from = smem + buf * kStage;
        intx4 x[UM], w[UN];
#pragma unroll
        for (int j = 0; j < UN; ++j) w[j] = *reinterpret_cast<const intx4*>(from + w_at + j * 1024);
#pragma unroll
        for (int i = 0; i < UM; ++i) x[i] = *reinterpret_cast<const intx4*>(from + x_at + i * 1024);
#pragma unroll
        for (int i = 0; i < UM; ++i)
#pragma unroll
            for (int j = 0; j < UN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[i], acc[i][j], 0, 0, 0);
        buf = buf + 1 == STAGES ? 0 : buf + 1;
        next = next + 1 == STAGES ? 0 : next + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the loads behind the last stage end before the workgroup does
    const bool vec = P.cout % 4 == 0 && reinterpret_cast<uintptr_t>(P.out) % (4 * sizeof(T)) == 0;
#pragma unroll
    for (int j = 0; j < UN; ++j) {
        const int o = o0 + (wn * UN + j) * 16 + g * 4;
        if (o >= P.cout) continue;
        floatx4 sw, bias{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = min(o + e, P.cout - 1);
            sw[e] = P.sw[c];
            if (P.bias) bias[e] = P.bias[c];
        }
#pragma unroll
        for (int i = 0; i < UM; ++i) {
            const int row = (m0 + wm * UM + i) * 16 + l16;
            if (row >= P.n_rows) continue;
            const float sx = P.sx[row];
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

template <typename T, int MT, int NT, int WM, int WN, int STAGES, bool W_TILED>
hipError_t gemm_launch(const FcI8& P, hipStream_t st) {
    constexpr unsigned lds = STAGES * (MT + NT) * 1024;
    auto kernel = fc_i8_gemm_kernel<T, MT, NT, WM, WN, STAGES, W_TILED>;
    static std::atomic<bool> raised{false};      // per instantiation
    if (lds > 64 * 1024 && !raised.load()) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        raised.store(true);
    }
    const size_t wgs = ((size_t)P.n_rows + MT * 16 - 1) / (MT * 16) * (((size_t)P.cout + NT * 16 - 1) / (NT * 16));
    if (wgs > 0x7fffffffu) return hipErrorInvalidValue;
    hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(WM * WN * 64), lds, st, P);
    return hipGetLastError();
}
template <typename T, int MT, int NT, int WM, int WN, int STAGES>
hipError_t gemm(const FcI8& P, bool w_tiled, hipStream_t st) {
    return w_tiled ? gemm_launch<T, MT, NT, WM, WN, STAGES, true>(P, st) : gemm_launch<T, MT, NT, WM, WN, STAGES, false>(P, st);
}

// [cout][K] -> tiles, K padded with zeros, the last tile's missing rows left out
__global__ __launch_bounds__(256) void tile_weights_kernel(const int8_t* __restrict__ w, int8_t* __restrict__ tiles, int K, int n_tiles, int cout) {
    const int piece = (blockIdx.x * 256 + threadIdx.x) >> 4, r = blockIdx.y * 16 + (threadIdx.x & 15);
    if (piece >= n_tiles * 4 || r >= cout) return;
    *reinterpret_cast<intx4*>(tiles + tile_offset(r, piece * 16, n_tiles)) = weights16(w + (size_t)r * K, piece * 16, K);
}

template <typename T>
hipError_t product(const FcI8& P, int8_t* w_tiles, hipStream_t st) {
    const dim3 block(kI8Waves * 64);
    const unsigned gx = (unsigned)((P.cout + 15) / 16);
    if (P.n_rows <= 16)
        hipLaunchKernelGGL((fc_i8_rows_kernel<T, 1>), dim3(gx, 1), block, 0, st, P);
    else if (P.n_rows <= kI8FewRows)
        hipLaunchKernelGGL((fc_i8_rows_kernel<T, 4>), dim3(gx, 1), block, 0, st, P);
    else {
        FcI8 Q = P;
        if (w_tiles) {
            hipLaunchKernelGGL(tile_weights_kernel, dim3((unsigned)((P.n_tiles * 4 + 15) / 16), gx), dim3(256), 0, st, P.w, w_tiles, P.K, P.n_tiles, P.cout);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            Q.w = w_tiles;
        }
        const long big = ((long)P.n_rows + 255) / 256 * ((P.cout + 255) / 256), mid = ((long)P.n_rows + 127) / 128 * ((P.cout + 127) / 128);
        if (big >= 192) return gemm<T, 16, 16, 2, 4, 4>(Q, w_tiles != nullptr, st);
        if (mid >= 192) return gemm<T, 8, 8, 2, 2, 4>(Q, w_tiles != nullptr, st);
        return gemm<T, 4, 4, 2, 2, 4>(Q, w_tiles != nullptr, st);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int dtype, size_t n_rows, int K, int8_t* q, float* scales, hipStream_t st) {
    return dtype == DC_BF16 ? quantize<__hip_bfloat16, false>((const __hip_bfloat16*)x, n_rows, K, q, scales, st)
                            : quantize<float, false>((const float*)x, n_rows, K, q, scales, st);
}

// The workspace: the rows in tiles, their scales, the weights in tiles.
struct I8Space { size_t rows, scales, weights, end; };
static I8Space i8_space(int n_rows, int K, int cout) {
    const size_t row = ((size_t)K + 63) / 64 * 64;
    I8Space s;
    s.rows = 0;
    s.scales = align_up(align_up(n_rows, 16) * row, 256);
    s.weights = s.scales + align_up((size_t)n_rows * sizeof(float), 256);
    s.end = s.weights + (n_rows > kI8FewRows ? align_up(align_up(cout, 16) * row, 256) : 0);
    return s;
}
size_t fc_i8_workspace(int n_rows, int K, int cout) { return i8_space(n_rows, K, cout).end; }

hipError_t launch_fc_i8(const void* x, const int8_t* w, const float* sw, const float* bias, void* out, int n_rows, int K, int cout, int relu,
                        int dtype, void* ws, hipStream_t st) {
    FcI8 P;
    P.n_rows = n_rows; P.K = K; P.n_tiles = (K + 63) / 64; P.cout = cout; P.relu = relu;
    const I8Space space = i8_space(n_rows, K, cout);
    int8_t* const base = static_cast<int8_t*>(ws);
    float* const sx = reinterpret_cast<float*>(base + space.scales);
    P.xq = base; P.sx = sx; P.w = w; P.sw = sw; P.bias = bias; P.out = out;
    const hipError_t e = dtype == DC_BF16 ? quantize<__hip_bfloat16, true>((const __hip_bfloat16*)x, n_rows, K, base, sx, st)
                                          : quantize<float, true>((const float*)x, n_rows, K, base, sx, st);
    if (e != hipSuccess) return e;
    const bool whole = K % 16 == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0;
    int8_t* const w_tiles = whole ? nullptr : base + space.weights;
    return dtype == DC_BF16 ? product<__hip_bfloat16>(P, w_tiles, st) : product<float>(P, w_tiles, st);
}

}  // namespace dc

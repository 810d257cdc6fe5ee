// Products in 8-bit integers: out[m][n] = act(x_scale[m] w_scale[n] sum_k q[m][k] w[n][k] + bias[n]), the sum in
// 32-bit integers on the matrix cores, and the steps q and their scales from rows of values.
#include <algorithm>
#include <type_traits>

#include "mpm_act.h"
#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// ---- values to steps ---------------------------------------------------------------------

constexpr float kSteps = 127.0f;
constexpr float kLeastScale = 0x1p-126f;

// A row's scale from the bits of its largest magnitude (as integers, NaN and infinity compare largest), and what
// turns its values into steps.
struct Steps {
    float scale;   // as stored
    float up;      // values and scale times this: away from the subnormal numbers
    float s, inv;  // the scale so raised, and about 1 / it

    __device__ __forceinline__ explicit Steps(uint32_t largest)
    {
        scale = fmaxf(__uint_as_float(largest) / kSteps, kLeastScale);
        up = scale < 0x1p-60f ? 0x1p64f : 1.0f;
        s = scale * up;
        inv = __builtin_amdgcn_rcpf(s);
        if (largest >= 0x7f800000u) scale = __uint_as_float(0x7fc00000u);
    }
    __device__ __forceinline__ bool finite() const { return scale == scale; }

    // x / s rounded to nearest even, of the real quotient: the product with the reciprocal is within a few
    // 2^-17 of it; next to a half the sign of x - (q +- 1/2) s decides, which one multiply-add gives exactly.
    __device__ __forceinline__ int of(float x) const
    {
        x *= up;
        const float r = x * inv;
        float q = __builtin_rintf(r);
        if (fabsf(r - q) > 0.5f - 0x1p-12f) {
            const float above = fmaf(-(q + 0.5f), s, x), below = fmaf(-(q - 0.5f), s, x);
            const bool odd = (int)q & 1;
            if (above > 0.0f || (above == 0.0f && odd)) q += 1.0f;
            else if (below < 0.0f || (below == 0.0f && odd)) q -= 1.0f;
        }
        return (int)fminf(fmaxf(q, -kSteps), kSteps);
    }
};

// The values of one vector of 16 bytes.
template <class S>
__device__ __forceinline__ float value(const u32x4& w, int e)
{
    if constexpr (S::kBytes == 2) return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
    return __uint_as_float(w[e]);
}

template <class S>
__device__ __forceinline__ uint32_t largest(const u32x4& w, uint32_t m)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (S::kBytes == 2) {
            m = max(m, (w[e] & 0x7fffu) << 16);
            m = max(m, w[e] & 0x7fff0000u);
        } else {
            m = max(m, w[e] & 0x7fffffffu);
        }
    }
    return m;
}

// The steps of one vector, a byte each, in words of four (bfloat16: two words, float32: one).
template <class S>
__device__ __forceinline__ void steps_of(const u32x4& w, const Steps& st, uint32_t (&out)[16 / S::kBytes / 4])
{
#pragma unroll
    for (int i = 0; i < 16 / S::kBytes / 4; ++i) {
        out[i] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (st.finite()) out[i] |= ((uint32_t)st.of(value<S>(w, 4 * i + e)) & 0xffu) << (8 * e);
    }
}

template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t m)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

constexpr int kQuantThreads = 256;

// Rows of at most VPL vectors a lane, a wave each, kept in registers between the maximum and the steps.
template <class S, int VPL>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(const uint8_t* __restrict__ x, long R, int K, long x_row,
                                                                 uint8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int kPer = 16 / S::kBytes, kWords = kPer / 4;
    const int lane = threadIdx.x % kWave, vecs = K / kPer, Kp = steps_row(K);
    const long row = (long)blockIdx.x * (kQuantThreads / kWave) + threadIdx.x / kWave;
    if (row >= R) return;
    const uint8_t* from = x + row * x_row * S::kBytes;
    u32x4 v[VPL];
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < VPL; ++u) v[u] = load16(from + (long)min(lane + u * kWave, vecs - 1) * 16);
#pragma unroll
    for (int u = 0; u < VPL; ++u) m = largest<S>(v[u], m);
    const Steps st(lanes_max<kWave>(m));
    if (lane == 0) scale[row] = st.scale;
    uint8_t* to = q + row * Kp;
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
        const int c = lane + u * kWave;
        if (c * kPer >= Kp) break;
        uint32_t w[kWords];
        steps_of<S>(v[u], st, w);
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint32_t*>(to + c * kPer)[i] = c < vecs ? w[i] : 0;
    }
}

// Wider rows: a workgroup each, read twice.
template <class S>
__global__ __launch_bounds__(kQuantThreads) void quantize_wide_kernel(const uint8_t* __restrict__ x, int K, long x_row,
                                                                      uint8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int kPer = 16 / S::kBytes, kWords = kPer / 4, kWaves = kQuantThreads / kWave;
    __shared__ uint32_t lds[kWaves];
    const int vecs = K / kPer, Kp = steps_row(K);
    const long row = blockIdx.x;
    const uint8_t* from = x + row * x_row * S::kBytes;
    uint32_t m = 0;
#pragma unroll 4
    for (int c = threadIdx.x; c < vecs; c += kQuantThreads) m = largest<S>(load16(from + (long)c * 16), m);
    m = lanes_max<kWave>(m);
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = m;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) m = max(m, lds[w]);
    const Steps st(m);
    if (threadIdx.x == 0) scale[row] = st.scale;
    uint8_t* to = q + row * Kp;
    for (int c = threadIdx.x; c * kPer < Kp; c += kQuantThreads) {
        uint32_t w[kWords];
        steps_of<S>(load16(from + (long)min(c, vecs - 1) * 16), st, w);
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint32_t*>(to + c * kPer)[i] = c < vecs ? w[i] : 0;
    }
}

template <class S>
hipError_t quantize(const uint8_t* x, long R, int K, long x_row, uint8_t* q, float* scale, hipStream_t st)
{
    constexpr int kPer = 16 / S::kBytes, kRows = kQuantThreads / kWave;
    const int vecs = steps_row(K) / kPer;
    const dim3 grid((unsigned)((R + kRows - 1) / kRows)), threads(kQuantThreads);
    if (vecs <= kWave) hipLaunchKernelGGL((quantize_kernel<S, 1>), grid, threads, 0, st, x, R, K, x_row, q, scale);
    else if (vecs <= 2 * kWave) hipLaunchKernelGGL((quantize_kernel<S, 2>), grid, threads, 0, st, x, R, K, x_row, q, scale);
    else if (vecs <= 4 * kWave) hipLaunchKernelGGL((quantize_kernel<S, 4>), grid, threads, 0, st, x, R, K, x_row, q, scale);
    else if (vecs <= 8 * kWave) hipLaunchKernelGGL((quantize_kernel<S, 8>), grid, threads, 0, st, x, R, K, x_row, q, scale);
    else hipLaunchKernelGGL((quantize_wide_kernel<S>), dim3((unsigned)R), threads, 0, st, x, K, x_row, q, scale);
    return hipGetLastError();
}

// ---- the end of a product ----------------------------------------------------------------

template <class T>
__device__ __forceinline__ float element(const void* p, long i)
{
    if constexpr (T::kBytes == 2) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
    return static_cast<const float*>(p)[i];
}
template <class T>
__device__ __forceinline__ void store_element(void* p, long i, float v)
{
    if constexpr (T::kBytes == 2) static_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_rne(v);
    else static_cast<float*>(p)[i] = v;
}

// The scales as they are multiplied: a sum of up to 2^30 times a token's scale of up to 2^121 stays finite, and the
// channel's takes the factor back (exact, but for token scales below 2^-102).
constexpr float kDown = 0x1p-24f, kUp = 0x1p24f;

template <class T, int ACT>
__device__ __forceinline__ float finish(int sum, float x_scale, float w_scale, float bias)
{
    return activate<ACT, T::kBytes == 4>(fmaf((float)sum * x_scale, w_scale, bias));
}

// ---- few tokens --------------------------------------------------------------------------

constexpr int kFew = 16;             // tokens
constexpr int kFewThreads = 256;
constexpr int kFewLds = 48 << 10;    // most bytes of steps made inside the product

struct Int8 {};

// A workgroup takes 16 output channels of all tokens, its waves every fourth 64 values of k. X: the type of x; values
// become steps in LDS first, in every workgroup by itself.
template <class X, class T, int ACT>
__global__ __launch_bounds__(kFewThreads) void few_kernel(Linear8Call a, const uint8_t* __restrict__ x, void* __restrict__ out)
{
    constexpr bool kValues = !std::is_same<X, Int8>::value;
    constexpr int kWaves = kFewThreads / kWave;
    extern __shared__ __align__(16) uint8_t q[];
    __shared__ int sums[kWaves][kFew * 16];
    __shared__ float scales[kFew];
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, M = (int)a.M, Kp = steps_row(a.K);
    const int n0 = blockIdx.x * 16, row = lane % 16, part = lane / 16;
    const int8_t* w = a.w + (long)min(n0 + row, a.N - 1) * Kp;
    if constexpr (kValues) {
        constexpr int kPer = 16 / X::kBytes, kWords = kPer / 4;
        for (int r = wave; r < M; r += kWaves) {
            const uint8_t* from = x + (long)r * a.x_row * X::kBytes;
            const int vecs = a.K / kPer;
            uint32_t m = 0;
            for (int c = lane; c < vecs; c += kWave) m = largest<X>(load16(from + c * 16), m);
            const Steps st(lanes_max<kWave>(m));
            if (lane == 0) scales[r] = st.scale;
            for (int c = lane; c * kPer < Kp; c += kWave) {
                uint32_t s[kWords];
                steps_of<X>(load16(from + min(c, vecs - 1) * 16), st, s);
#pragma unroll
                for (int i = 0; i < kWords; ++i) reinterpret_cast<uint32_t*>(q + r * Kp + c * kPer)[i] = c < vecs ? s[i] : 0;
            }
        }
    } else {
        if (t < M) scales[t] = a.x_scale[t];
    }
    __syncthreads();
    i32x4 acc = {0, 0, 0, 0};
    const i32x4 none = {0, 0, 0, 0};
    for (int k = wave * 64; k < Kp; k += kWaves * 64) {
        const int at = k + part * 16;
        const bool in = at < Kp;
        const i32x4 wv = *reinterpret_cast<const i32x4*>(w + (in ? at : 0));
        i32x4 xv = none;
        if (in && row < M) {
            if constexpr (kValues) xv = *reinterpret_cast<const i32x4*>(q + row * Kp + at);
            else xv = *reinterpret_cast<const i32x4*>(x + (long)row * Kp + at);
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc, 0, 0, 0);
    }
    // acc[r]: channel 4 part + r of token `row`.
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][row * 16 + 4 * part + r] = acc[r];
    __syncthreads();
    const int m = t / 16, n = n0 + t % 16;
    if (m >= M || n >= a.N) return;
    int s = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) s += sums[i][t];
    const float bias = a.bias ? element<T>(a.bias, n) : 0.0f;
    store_element<T>(out, (long)m * a.out_row + n, finish<T, ACT>(s, scales[m] * kDown, a.w_scale[n] * kUp, bias));
}

// ---- many tokens -------------------------------------------------------------------------

constexpr int kXcds = 8;  // workgroups are dealt round-robin to 8 XCDs, each with its own L2

// Workgroup barrier that waits only for this wave's LDS operations, not for loads on their way to LDS.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A workgroup computes BM tokens x BN channels with WM x WN waves, k in steps of BK bytes through STAGES LDS buffers that
// loads fill directly. A buffer holds rows of BK bytes, BM of tokens and then BN of weights, the 16-byte pieces of a row
// in an order of its own (piece c of row r at place c ^ swizzle(r)), so that the 32 rows of a fragment are read
// without bank conflicts; the loads bring each lane's piece from where that order has it.
template <int BM, int BN, int WM, int WN, int BK, int STAGES, class T, int ACT>
__global__ __launch_bounds__(WM* WN* kWave, 2) void product_kernel(Linear8Call a, const uint8_t* __restrict__ q,
                                                                const float* __restrict__ q_scale, void* __restrict__ out,
                                                                int mtiles, int ntiles, bool whole)
{
    constexpr int kWaves = WM * WN, THREADS = kWaves * kWave;
    constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
    constexpr int kPieces = BK / 16;              // of a row
    constexpr int kRows = kWave / kPieces;        // rows a load instruction of a wave brings
    constexpr int kStage = (BM + BN) * BK;
    constexpr int kLoads = (BM + BN) / kRows / kWaves;
    static_assert((BM + BN) % (kRows * kWaves) == 0 && BM % kRows == 0, "whole loads");
    constexpr int kSteps32 = BK / 32;
    extern __shared__ __align__(1024) uint8_t lds[];
    float* w_scale = reinterpret_cast<float*>(lds + STAGES * kStage);
    float* bias = w_scale + BN;

    // Tiles in order, tokens outside, dealt to the XCDs in eight contiguous shares.
    const long tiles = (long)mtiles * ntiles;
    const int xcd = blockIdx.x % kXcds;
    const long tile = tiles * xcd / kXcds + blockIdx.x / kXcds;
    if (tile >= tiles * (xcd + 1) / kXcds) return;
    const long m0 = tile / ntiles * BM;
    const int n0 = (int)(tile % ntiles) * BN;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, half = lane >> 5;
    const int wm = wave % WM, wn = wave / WM;
    const int Kp = steps_row(a.K), chunks = (Kp + BK - 1) / BK;

    for (int i = t; i < BN; i += THREADS) {
        const int n = min(n0 + i, a.N - 1);
        w_scale[i] = a.w_scale[n] * kUp;
        bias[i] = a.bias ? element<T>(a.bias, n) : 0.0f;
    }

    auto swizzle = [](int row) { return kPieces == 8 ? row & 7 : (row >> 1) & 3; };
    // This lane's rows and pieces: load i of wave w brings rows (w + kWaves i) kRows ... of the buffer.
    const uint8_t* from[kLoads];
    const int lrow = lane / kPieces, piece = (lane % kPieces) ^ swizzle(lrow);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = (wave + kWaves * i) * kRows + lrow;  // (kRows and BM are multiples of 8: the swizzle is lrow's)
        from[i] = r < BM ? q + min(m0 + r, a.M - 1) * Kp
                         : reinterpret_cast<const uint8_t*>(a.w) + (long)min(n0 + r - BM, a.N - 1) * Kp;
    }
    auto issue = [&](int chunk, int i) {
        // Past a row's end the last piece again: the products leave it out.
        const uint8_t* p = from[i] + min(chunk * BK + piece * 16, Kp - 16);
        const uint32_t to = (uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)(
            lds + (chunk % STAGES) * kStage + (wave + kWaves * i) * kRows * BK);
        asm volatile("global_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(to) : "memory");
    };
    const int sw = swizzle(l32);
    i32x16 acc[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = i32x16{};
    i32x4 fw[2][NT], fx[2][MT];
    auto read = [&](int to, int chunk, int g) {
        const uint8_t* s = lds + (chunk % STAGES) * kStage + l32 * BK + (((2 * g + half) ^ sw) << 4);
#pragma unroll
        for (int m = 0; m < MT; ++m) fx[to][m] = *reinterpret_cast<const i32x4*>(s + (wm * MT + m) * 32 * BK);
#pragma unroll
        for (int n = 0; n < NT; ++n) fw[to][n] = *reinterpret_cast<const i32x4*>(s + (BM + (wn * NT + n) * 32) * BK);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m)
                acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[from][n], fx[from][m], acc[n][m], 0, 0, 0);
    };

#pragma unroll
    for (int c = 0; c < STAGES - 1; ++c)
        if (c < chunks) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) issue(c, i);
        }
    const int full = Kp / BK;
    for (int c = 0; c < chunks; ++c) {
        // The loads of chunk c are done when at most those of the chunks after it are on their way.
        if (c + STAGES - 2 < chunks) wait_loads<kLoads*(STAGES - 2)>();
        else wait_loads<0>();
        lds_barrier();
        if (c + STAGES - 1 < chunks) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) issue(c + STAGES - 1, i);
        }
        if (c < full) {
            read(0, c, 0);
#pragma unroll
            for (int g = 0; g < kSteps32; ++g) {
                if (g + 1 < kSteps32) read((g + 1) & 1, c, g + 1);
                multiply(g & 1);
            }
        } else {
            const int left = Kp - c * BK;
            for (int g = 0; g * 32 < left; ++g) {
                read(0, c, g);
                if (g * 32 + 16 >= left && half) {  // the second 16 bytes lie past the end
                    const i32x4 none = {0, 0, 0, 0};
#pragma unroll
                    for (int m = 0; m < MT; ++m) fx[0][m] = none;
                }
                multiply(0);
            }
        }
    }

    // acc[n][m][r]: token m * 32 + l32 of the wave's, channel n * 32 + 8 (r / 4) + 4 half + r % 4.
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const long row = m0 + (wm * MT + m) * 32 + l32;
        const float xs = q_scale[min(row, a.M - 1)] * kDown;
        const bool live = row < a.M;
        uint8_t* to = static_cast<uint8_t*>(out) + row * a.out_row * T::kBytes;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int nb = (wn * NT + n) * 32;
            float v[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = nb + 8 * (r / 4) + 4 * half + r % 4;
                v[r] = finish<T, ACT>(acc[n][m][r], xs, w_scale[i], bias[i]);
            }
            if (whole) {
                if constexpr (T::kBytes == 4) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int i = n0 + nb + 8 * c + 4 * half;
                        const u32x4 w = {__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]),
                                         __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3])};
                        if (live && i < a.N) store16(to + i * 4L, w);
                    }
                } else {
                    // Half a wave exchanges channels with the other, so that a lane has eight in a row.
#pragma unroll
                    for (int c = 0; c < 4; c += 2) {
                        uint32_t w[2][2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            typedef float f32x2 __attribute__((ext_vector_type(2)));
                            const f32x2 p = {v[4 * c + 2 * e], v[4 * c + 2 * e + 1]};
                            const f32x2 s = {v[4 * c + 4 + 2 * e], v[4 * c + 5 + 2 * e]};
                            const auto x = __builtin_amdgcn_permlane32_swap(
                                __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2)),
                                __builtin_bit_cast(uint32_t, __builtin_convertvector(s, bf16x2)), false, false);
                            w[0][e] = x[0];
                            w[1][e] = x[1];
                        }
                        const u32x4 packed = {w[0][0], w[0][1], w[1][0], w[1][1]};
                        const int i = n0 + nb + 8 * (c + half);
                        if (live && i < a.N) store16(to + i * 2L, packed);
                    }
                }
            } else if (live) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = n0 + nb + 8 * (r / 4) + 4 * half + r % 4;
                    if (i < a.N) store_element<T>(to, i, v[r]);
                }
            }
        }
    }
}

template <int BM, int BN, int WM, int WN, int BK, int STAGES, class T, int ACT>
hipError_t product(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t st)
{
    constexpr size_t bytes = (size_t)STAGES * (BM + BN) * BK + 2 * BN * 4;
    const auto kernel = product_kernel<BM, BN, WM, WN, BK, STAGES, T, ACT>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    const long mtiles = (a.M + BM - 1) / BM, ntiles = (a.N + BN - 1) / BN, per = (mtiles * ntiles + kXcds - 1) / kXcds;
    // Rows of whole 16 bytes, of a whole number of them: written 16 bytes at a time.
    constexpr int kPer = 16 / T::kBytes;
    const bool whole = a.N % kPer == 0 && a.out_row % kPer == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(per * kXcds)), dim3(WM * WN * kWave), bytes, st, a,
                       reinterpret_cast<const uint8_t*>(q), q_scale, out, (int)mtiles, (int)ntiles, whole);
    return hipGetLastError();
}

template <class T, int ACT>
hipError_t product_of(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t st)
{
    const long big = ((a.M + 127) / 128) * ((a.N + 255) / 256);
    if (big >= 256) return product<128, 256, 2, 2, 64, 3, T, ACT>(a, q, q_scale, out, st);
    return product<64, 64, 2, 2, 128, 3, T, ACT>(a, q, q_scale, out, st);
}

// Calls go(output type, activation).
template <class F>
hipError_t with_kind(const Linear8Call& a, F&& go)
{
    auto act = [&](auto type) {
        switch (a.act) {
        case kActRelu: return go(type, std::integral_constant<int, kActRelu>{});
        case kActSilu: return go(type, std::integral_constant<int, kActSilu>{});
        case kActGelu: return go(type, std::integral_constant<int, kActGelu>{});
        default: return go(type, std::integral_constant<int, kActNone>{});
        }
    };
    return a.dt == kBf16 ? act(Bf16{}) : act(F32{});
}

}  // namespace

hipError_t launch_quantize(const void* x, long R, int K, long x_row, int dt, int8_t* q, float* scale, hipStream_t stream)
{
    const uint8_t* xp = static_cast<const uint8_t*>(x);
    uint8_t* qp = reinterpret_cast<uint8_t*>(q);
    return dt == kBf16 ? quantize<Bf16>(xp, R, K, x_row, qp, scale, stream)
                       : quantize<F32>(xp, R, K, x_row, qp, scale, stream);
}

bool linear8_is_few(const Linear8Call& a)
{
    return a.M <= kFew && (a.x_dt == kI8 || a.M * steps_row(a.K) <= kFewLds);
}

hipError_t launch_linear8_few(const Linear8Call& a, const void* x, void* out, hipStream_t stream)
{
    const uint8_t* xp = static_cast<const uint8_t*>(x);
    const dim3 grid((unsigned)((a.N + 15) / 16)), threads(kFewThreads);
    const size_t bytes = a.x_dt == kI8 ? 0 : (size_t)a.M * steps_row(a.K);
    return with_kind(a, [&](auto type, auto act) {
        typedef decltype(type) T;
        constexpr int ACT = decltype(act)::value;
        if (a.x_dt == kI8) hipLaunchKernelGGL((few_kernel<Int8, T, ACT>), grid, threads, bytes, stream, a, xp, out);
        else if (a.x_dt == kBf16) hipLaunchKernelGGL((few_kernel<Bf16, T, ACT>), grid, threads, bytes, stream, a, xp, out);
        else hipLaunchKernelGGL((few_kernel<F32, T, ACT>), grid, threads, bytes, stream, a, xp, out);
        return hipGetLastError();
    });
}

hipError_t launch_linear8(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t stream)
{
    return with_kind(a, [&](auto type, auto act) {
        return product_of<decltype(type), decltype(act)::value>(a, q, q_scale, out, stream);
    });
}

}  // namespace mpm

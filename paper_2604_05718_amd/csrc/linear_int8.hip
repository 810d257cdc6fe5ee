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

constexpr int kUnits = 256;  // compute units
constexpr int kXcds = 8;     // workgroups are dealt round-robin to 8 XCDs, each with its own L2

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

// Writes 32 channels' results of one token, channels `at` + 8 (r / 4) + 4 half + r % 4 in v[r], those
// below N. `whole`: 16 bytes at a time.
template <class T>
__device__ __forceinline__ void write_row(uint8_t* to, int at, int half, int N, bool whole, const float (&v)[16])
{
    if (!whole) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int i = at + 8 * (r / 4) + 4 * half + r % 4;
            if (i < N) store_element<T>(to, i, v[r]);
        }
        return;
    }
    if constexpr (T::kBytes == 4) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int i = at + 8 * c + 4 * half;
            const u32x4 w = {__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]),
                             __float_as_uint(v[4 * c + 3])};
            if (i < N) store16(to + i * 4L, w);
        }
    } else {
        // Half a wave exchanges channels with the other, so that a lane has eight in a row.
        auto pair = [&](int r) {
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            const f32x2 p = {v[r], v[r + 1]};
            return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        };
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
            const auto x = __builtin_amdgcn_permlane32_swap(pair(4 * c), pair(4 * c + 4), false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(pair(4 * c + 2), pair(4 * c + 6), false, false);
            const u32x4 w = {x[0], y[0], x[1], y[1]};
            const int i = at + 8 * (c + half);
            if (i < N) store16(to + i * 2L, w);
        }
    }
}

// What a workgroup takes of the tiles: those of its XCD's contiguous share (tokens outside, channels inside), `slots`
// workgroups by turns.
struct Share {
    long tile, end;
    int slots;
};
__device__ __forceinline__ Share share(long tiles)
{
    const int xcd = blockIdx.x % kXcds;
    return Share{tiles * xcd / kXcds + blockIdx.x / kXcds, tiles * (xcd + 1) / kXcds, (int)(gridDim.x / kXcds)};
}

// Tiles of BM tokens x BN channels, WM x WN waves, k in chunks of BK bytes through STAGES LDS buffers that loads fill
// directly. A buffer holds rows of BK bytes, BM of tokens and then BN of weights, the 16-byte pieces of a row in an
// order of its own (piece c of row r at place c ^ swizzle(r)), so that the 32 rows of a fragment are read
// without bank conflicts; the loads bring each lane's piece from where that order has it. A workgroup walks its
// tiles with the chunks of all of them as one stream, loads STAGES - 1 chunks ahead, also behind a tile's end: the
// next tile's first chunks arrive while this one's results are finished, and those are written while the next
// one's products run.
template <int BM, int BN, int WM, int WN, int BK, int STAGES, class T, int ACT>
__global__ __launch_bounds__(WM* WN* kWave, 2) void product_kernel(Linear8Call a, const uint8_t* __restrict__ q,
                                                                   const float* __restrict__ q_scale,
                                                                   void* __restrict__ out, int mtiles, int ntiles, bool whole)
{
    constexpr int kWaves = WM * WN, THREADS = kWaves * kWave;
    constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
    constexpr int kPieces = BK / 16;              // of a row
    constexpr int kRows = kWave / kPieces;        // rows a load instruction of a wave brings
    constexpr int kStage = (BM + BN) * BK;
    constexpr int kLoads = (BM + BN) / kRows / kWaves;
    constexpr int kSteps32 = BK / 32;
    constexpr int kAhead = STAGES - 1;
    static_assert((BM + BN) % (kRows * kWaves) == 0 && BM % kRows == 0, "whole loads");
    // (A wave's loads are a whole number of 16 rows apart, so a lane's swizzle is one for all.)
    static_assert(kRows * kWaves % 16 == 0 && BM % 16 == 0, "one swizzle a lane");
    static_assert(BN <= THREADS && BM + BN <= 2 * THREADS, "scales: a thread each");
    extern __shared__ __align__(1024) uint8_t lds[];
    float* channels = reinterpret_cast<float*>(lds + STAGES * kStage);  // [2][scale, bias][BN], by tiles in turns

    const Share sh = share((long)mtiles * ntiles);
    if (sh.tile >= sh.end) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, half = lane >> 5;
    const int wm = wave % WM, wn = wave / WM;
    const int Kp = steps_row(a.K), chunks = (Kp + BK - 1) / BK, full = Kp / BK;

    // 16 rows of one piece meet the 64 banks once.
    auto swizzle = [](int row) { return kPieces == 8 ? (row >> 1) & 7 : (row >> 2) & 3; };
    // The stream's end that loads: its tile and chunk, and this lane's rows there (load i of a wave brings rows
    // (wave + kWaves i) kRows ... of the buffer), clamped to those that exist.
    const int lrow = lane / kPieces, piece = ((lane % kPieces) ^ swizzle(wave * kRows + lrow)) * 16;
    const uint8_t* from[kLoads];
    long ltile = sh.tile;
    int lchunk = 0, lbuf = 0;
    auto place = [&](long tile) {
        const long m0 = tile / ntiles * BM;
        const int n0 = (int)(tile % ntiles) * BN;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = (wave + kWaves * i) * kRows + lrow;
            from[i] = r < BM ? q + min(m0 + r, a.M - 1) * Kp
                             : reinterpret_cast<const uint8_t*>(a.w) + (long)min(n0 + r - BM, a.N - 1) * Kp;
        }
    };
    // The scales of a tile: a lane's tokens', and a thread's channel's on its way to LDS.
    float xs[MT], w_scale, bias;
    auto load_scales = [&](long tile) {
        const long m0 = tile / ntiles * BM;
        const int n = min((int)(tile % ntiles) * BN + min(t, BN - 1), a.N - 1);
#pragma unroll
        for (int m = 0; m < MT; ++m) xs[m] = q_scale[min(m0 + (wm * MT + m) * 32 + l32, a.M - 1)] * kDown;
        w_scale = a.w_scale[n] * kUp;
        bias = a.bias ? element<T>(a.bias, n) : 0.0f;
    };
    // The next chunk of the stream, if there is one.
    auto issue = [&]() {
        if (ltile >= sh.end) return;
        const uint32_t to = (uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)(
            lds + lbuf * kStage + wave * kRows * BK);
        // Past a row's end the last piece again: the products leave it out.
        const int at = min(lchunk * BK + piece, Kp - 16);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            asm volatile("global_load_lds_dwordx4 %0, off" ::"v"(from[i] + at), "{m0}"(to + kWaves * i * kRows * BK)
                         : "memory");
        lbuf = lbuf + 1 == STAGES ? 0 : lbuf + 1;
        if (++lchunk == chunks) {
            lchunk = 0;
            ltile += sh.slots;
            if (ltile < sh.end) place(ltile);
        }
    };

    const int sw = swizzle(l32);
    i32x16 acc[NT][MT];
    i32x4 fw[2][NT], fx[2][MT];
    int buf = 0;  // of the chunk that is multiplied
    auto read = [&](int to, int g) {
        const uint8_t* s = lds + buf * kStage + l32 * BK + (((2 * g + half) ^ sw) << 4);
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
    // Chunk c of a tile is there once at most the loads of the kAhead - 1 chunks behind it in the stream are on their
    // way (no count but 0 at the stream's end). A tile's first kAhead have been waited for before.
    auto arrive = [&](int c) {
        if (c >= kAhead) {
            if (ltile < sh.end) wait_loads<kLoads*(kAhead - 1)>();
            else wait_loads<0>();
        }
        lds_barrier();
        issue();
    };

    load_scales(sh.tile);
    place(sh.tile);
    for (int c = 0; c < kAhead; ++c) issue();
    wait_loads<0>();
    int turn = 0;
    auto hand_over = [&]() {  // the channels' values of the tile that comes
        if (t < BN) {
            channels[(2 * turn) * BN + t] = w_scale;
            channels[(2 * turn + 1) * BN + t] = bias;
        }
    };
    hand_over();
#pragma unroll 1
    for (long tile = sh.tile; tile < sh.end; tile += sh.slots) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[n][m] = i32x16{};
#pragma unroll 1
        for (int c = 0; c < full; ++c) {
            arrive(c);
            read(0, 0);
#pragma unroll
            for (int g = 0; g < kSteps32; ++g) {
                if (g + 1 < kSteps32) read((g + 1) & 1, g + 1);
                multiply(g & 1);
            }
            buf = buf + 1 == STAGES ? 0 : buf + 1;
        }
        if (full < chunks) {
            arrive(full);
            const int left = Kp - full * BK;
#pragma unroll 1
            for (int g = 0; g * 32 < left; ++g) {
                read(0, g);
                if (g * 32 + 16 >= left && half) {  // the second 16 bytes lie past the end
                    const i32x4 none = {0, 0, 0, 0};
#pragma unroll
                    for (int m = 0; m < MT; ++m) fx[0][m] = none;
                }
                multiply(0);
            }
            buf = buf + 1 == STAGES ? 0 : buf + 1;
        }

        // Everything on its way has arrived before the first write leaves, so that no wait for loads waits for writes.
        float now[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) now[m] = xs[m];
        const float *ws = channels + 2 * turn * BN, *bs = ws + BN;
        const bool last = tile + sh.slots >= sh.end;
        if (!last) load_scales(tile + sh.slots);
        wait_loads<0>();
        turn ^= 1;
        if (!last) hand_over();
        // acc[n][m][r]: token m * 32 + l32 of the wave's, channel n * 32 + 8 (r / 4) + 4 half + r % 4.
        const long m0 = tile / ntiles * BM;
        const int n0 = (int)(tile % ntiles) * BN;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const long row = m0 + (wm * MT + m) * 32 + l32;
            uint8_t* to = static_cast<uint8_t*>(out) + row * a.out_row * T::kBytes;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int nb = (wn * NT + n) * 32;
                float v[16];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const f32x4 w = *reinterpret_cast<const f32x4*>(ws + nb + 8 * c + 4 * half);
                    const f32x4 b = *reinterpret_cast<const f32x4*>(bs + nb + 8 * c + 4 * half);
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[4 * c + r] = finish<T, ACT>(acc[n][m][4 * c + r], now[m], w[r], b[r]);
                }
                if (row < a.M) write_row<T>(to, n0 + nb, half, a.N, whole, v);
            }
        }
    }
}

template <int BM, int BN, int WM, int WN, int BK, int STAGES, class T, int ACT>
hipError_t product(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t st)
{
    constexpr size_t bytes = (size_t)STAGES * (BM + BN) * BK + 4 * BN * 4;
    const auto kernel = product_kernel<BM, BN, WM, WN, BK, STAGES, T, ACT>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    const long mtiles = (a.M + BM - 1) / BM, ntiles = (a.N + BN - 1) / BN, per = (mtiles * ntiles + kXcds - 1) / kXcds;
    // As many workgroups as the chip holds (by LDS and by registers: two waves a SIMD).
    constexpr int kHeld = (int)std::min<size_t>((160 << 10) / bytes, 8 / (WM * WN) > 0 ? 8 / (WM * WN) : 1);
    const long slots = std::min(per, (long)kHeld * kUnits / kXcds);
    // Rows of whole 16 bytes, of a whole number of them: written 16 bytes at a time.
    constexpr int kPer = 16 / T::kBytes;
    const bool whole = a.N % kPer == 0 && a.out_row % kPer == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(slots * kXcds)), dim3(WM * WN * kWave), bytes, st, a,
                       reinterpret_cast<const uint8_t*>(q), q_scale, out, (int)mtiles, (int)ntiles, whole);
    return hipGetLastError();
}

// The widest tiles that leave no compute unit idle: a tile of 256 x 256 loads half the bytes a product that one of 128 x 128
// does, which loads half of what one of 64 x 64 does. Products (bfloat16 results, no activation) in tiles of 64 / 128 /
// 256, us: 4103 x 150 x 848 7.3 / 11.6 / 23, 512 x 768 x 768 5.1 / 7.4 / 15.1, 1024 x 2304 x 768 9.2 / 8.2 / 16.3,
// 8000 x 1024 x 1024 23.7 / 15.6 / 21.2, 11000 x 2304 x 768 49 / 33.1 / 34.0, 45888 x 2304 x 768 159 / 124 / 119.
template <class T, int ACT>
hipError_t product_of(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t st)
{
    auto tiles = [&](int rows) { return (a.M + rows - 1) / rows * ((a.N + rows - 1) / rows); };
    if (tiles(256) >= 2 * kUnits) return product<256, 256, 2, 4, 128, 2, T, ACT>(a, q, q_scale, out, st);
    if (tiles(128) >= kUnits / 2) return product<128, 128, 2, 2, 128, 2, T, ACT>(a, q, q_scale, out, st);
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

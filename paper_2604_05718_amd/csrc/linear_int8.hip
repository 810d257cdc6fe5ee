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

// The values of one vector of 16 bytes.
template <class S>
__device__ __forceinline__ float value(const u32x4& w, int e)
{
    if constexpr (S::kBytes == 2) return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
    return __uint_as_float(w[e]);
}

// The bits of the largest magnitude (as integers NaN and infinity compare largest).
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

// A row's scale, from the bits of its largest magnitude, and what turns its values into steps.
struct Steps {
    float scale, inv;  // as stored, and about 1 / it
    bool finite;

    __device__ __forceinline__ explicit Steps(uint32_t most)
    {
        const float s = fmaxf(__uint_as_float(most) / kSteps, kLeastScale);
        finite = most < 0x7f800000u;
        inv = __builtin_amdgcn_rcpf(s);
        scale = finite ? s : __uint_as_float(0x7fc00000u);
    }

    // x / scale rounded to nearest even, of the real quotient: next to a half the sign of x - (q +- 1/2) scale decides, which
    // one multiply-add gives exactly (raised where it could leave the numbers that float32 holds).
    __device__ __forceinline__ int exact(float x) const
    {
        const float up = scale < 0x1p-60f ? 0x1p64f : 1.0f, s = scale * up;
        float q = __builtin_rintf(x * inv);
        x *= up;
        const float above = fmaf(-(q + 0.5f), s, x), below = fmaf(-(q - 0.5f), s, x);
        const bool odd = (int)q & 1;
        if (above > 0.0f || (above == 0.0f && odd)) q += 1.0f;
        else if (below < 0.0f || (below == 0.0f && odd)) q -= 1.0f;
        return (int)q;
    }

    // The steps of one vector, a byte each, in words of four (bfloat16: two words, float32: one). The product with the
    // reciprocal is within 2^-15 of the quotient; adding 1.5 2^23 leaves its rounding in the sum's low bits.
    template <class S>
    __device__ __forceinline__ void of(const u32x4& w, uint32_t (&out)[16 / S::kBytes / 4]) const
    {
        constexpr float kMagic = 12582912.0f;
        constexpr int kPer = 16 / S::kBytes;
        uint32_t t[kPer];
        float off = 0.0f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float r = value<S>(w, e) * inv, m = r + kMagic;
            t[e] = __float_as_uint(m);
            off = fmaxf(off, fabsf(r - (m - kMagic)));
        }
        if (off > 0.5f - 0x1p-14f) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) t[e] = (uint32_t)exact(value<S>(w, e));
        }
#pragma unroll
        for (int i = 0; i < kPer / 4; ++i) {
            const uint32_t lo = __builtin_amdgcn_perm(t[4 * i + 1], t[4 * i], 0x0c0c0400u);
            const uint32_t hi = __builtin_amdgcn_perm(t[4 * i + 3], t[4 * i + 2], 0x0c0c0400u);
            out[i] = finite ? lo | hi << 16 : 0;
        }
    }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}

// The largest of a value over 32 or 64 lanes, in every lane (the exchanges of lanes_sum).
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    v = dpp_max<0xb1>(v);
    v = dpp_max<0x4e>(v);
    v = dpp_max<0x141>(v);
    v = dpp_max<0x140>(v);
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(p[0], p[1]);
    if constexpr (LANES >= kWave) {
        const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(q[0], q[1]);
    }
    return v;
}

constexpr int kQuantThreads = 256;
constexpr long kMostGroups = 1L << 22;  // workgroups of a launch (a grid holds 2^32 threads); they take further rows in turns

template <class S>
__device__ __forceinline__ void store_steps(uint8_t* to, const uint32_t (&w)[16 / S::kBytes / 4], bool in)
{
    if constexpr (S::kBytes == 2) {
        typedef uint32_t Two __attribute__((ext_vector_type(2)));
        const Two v = {in ? w[0] : 0, in ? w[1] : 0};
        *reinterpret_cast<Two*>(to) = v;
    } else {
        *reinterpret_cast<uint32_t*>(to) = in ? w[0] : 0;
    }
}

// Rows of at most VPL vectors a lane, LANES lanes each, kept in registers between the maximum and the steps.
// 45888 rows of 768 bfloat16 values (106 MB): 19 us, 5.6 TB/s.
template <class S, int LANES, int VPL>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(const uint8_t* __restrict__ x, long R, int K, long x_row,
                                                                 uint8_t* __restrict__ q, float* __restrict__ scale)
{
    constexpr int kPer = 16 / S::kBytes, kWords = kPer / 4;
    const int lane = threadIdx.x % LANES, vecs = K / kPer, Kp = steps_row(K);
    constexpr int kRows = kQuantThreads / LANES;
    for (long first = (long)blockIdx.x * kRows; first < R; first += (long)gridDim.x * kRows) {
        const long at = first + threadIdx.x / LANES, row = min(at, R - 1);
        const uint8_t* from = x + row * x_row * S::kBytes;
        u32x4 v[VPL];
        uint32_t m = 0;
#pragma unroll
        for (int u = 0; u < VPL; ++u) v[u] = load16(from + (long)min(lane + u * LANES, vecs - 1) * 16);
#pragma unroll
        for (int u = 0; u < VPL; ++u) m = largest<S>(v[u], m);
        const Steps st(lanes_max<LANES>(m));
        if (at >= R) return;
        if (lane == 0) scale[row] = st.scale;
        uint8_t* to = q + row * Kp;
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
            const int c = lane + u * LANES;
            if (c * kPer >= Kp) break;
            uint32_t w[kWords];
            st.of<S>(v[u], w);
            store_steps<S>(to + c * kPer, w, c < vecs);
        }
    }
}

// Wider rows, and few of more than two vectors a lane of half a wave: a workgroup each, read twice. us so / in half a wave or a
// wave each, bfloat16: 300 rows of 1024 values 3.3 / 6.3, 1000 3.6 / 5.4, 60 of 4096 4.8 / 7.7, 1000 7.0 / 10.9, of 2048 7.0 / 6.8.
// (Half a wave a row for many: 45888 of 192 10.4, in a wave each 16.9; of 768 19.4 and 23.9.)
constexpr int kFewRows = 1024;
template <class S>
__global__ __launch_bounds__(kQuantThreads) void quantize_wide_kernel(const uint8_t* __restrict__ x, long R, int K,
                                                                      long x_row, uint8_t* __restrict__ q,
                                                                      float* __restrict__ scale)
{
    constexpr int kPer = 16 / S::kBytes, kWords = kPer / 4, kWaves = kQuantThreads / kWave;
    __shared__ uint32_t lds[kWaves];
    const int vecs = K / kPer, Kp = steps_row(K);
    for (long row = blockIdx.x; row < R; row += gridDim.x) {
        const uint8_t* from = x + row * x_row * S::kBytes;
        uint32_t m = 0;
#pragma unroll 4
        for (int c = threadIdx.x; c < vecs; c += kQuantThreads) m = largest<S>(load16(from + (long)c * 16), m);
        m = lanes_max<kWave>(m);
        __syncthreads();  // the row before has been read
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = m;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) m = max(m, lds[w]);
        const Steps st(m);
        if (threadIdx.x == 0) scale[row] = st.scale;
        uint8_t* to = q + row * Kp;
        for (int c = threadIdx.x; c * kPer < Kp; c += kQuantThreads) {
            uint32_t w[kWords];
            st.of<S>(load16(from + (long)min(c, vecs - 1) * 16), w);
            store_steps<S>(to + c * kPer, w, c < vecs);
        }
    }
}

template <class S>
hipError_t quantize(const uint8_t* x, long R, int K, long x_row, uint8_t* q, float* scale, hipStream_t st)
{
    const int vecs = steps_row(K) / (16 / S::kBytes);
    auto rows = [&](auto lanes, auto vpl) {
        constexpr int L = decltype(lanes)::value, kRows = kQuantThreads / L;
        hipLaunchKernelGGL((quantize_kernel<S, L, decltype(vpl)::value>),
                           dim3((unsigned)std::min((R + kRows - 1) / kRows, kMostGroups)), dim3(kQuantThreads), 0, st, x, R, K,
                           x_row, q, scale);
    };
    constexpr std::integral_constant<int, 32> half{};
    constexpr std::integral_constant<int, kWave> wave{};
    if (vecs <= 32) rows(half, std::integral_constant<int, 1>{});
    else if (vecs <= 64) rows(half, std::integral_constant<int, 2>{});
    else if (vecs <= 96 && R > kFewRows) rows(half, std::integral_constant<int, 3>{});
    else if (vecs <= 128 && R > kFewRows) rows(half, std::integral_constant<int, 4>{});
    else if (vecs <= 256 && R > kFewRows) rows(wave, std::integral_constant<int, 4>{});
    else if (vecs <= 512 && R > kFewRows) rows(wave, std::integral_constant<int, 8>{});
    else hipLaunchKernelGGL((quantize_wide_kernel<S>), dim3((unsigned)std::min(R, kMostGroups)), dim3(kQuantThreads), 0, st, x, R,
                            K, x_row, q, scale);
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

constexpr int kFewLds = 32 << 10;  // most bytes of steps made inside the product
constexpr int kFewAhead = 4;       // pieces of 64 values a wave has on their way

struct Int8 {};

// A workgroup takes 16 output channels of 16 MT tokens, each of W waves every W-th piece of 64 values of k; the waves' sums
// meet in LDS. X: the type of x; values (16 tokens, at most W) become steps in LDS first, in every workgroup by itself, while
// the first weights are on their way: a wave has one row or a slice of one. What bounds it is the latency of one pass over
// its rows: from bfloat16 values to bfloat16 results, replayed without pauses, 1 x 2304 x 768 takes 3.9 us (W = 16 5.1), 16 x
// 4096 x 1024 7.4, 8 x 1024 x 4096 8.9 (W = 4 22.9, in tiles after quantising 19).
template <class X, class T, int ACT, int MT, int W>
__global__ __launch_bounds__(W* kWave) void few_kernel(Linear8Call a, const uint8_t* __restrict__ x, void* __restrict__ out)
{
    constexpr bool kValues = !std::is_same<X, Int8>::value;
    static_assert(!kValues || (MT == 1 && W <= 16), "a row has a wave");
    extern __shared__ __align__(16) uint8_t lds[];  // steps, then the waves' sums
    __shared__ float scales[16 * MT];
    __shared__ uint32_t most[kValues ? W : 1];
    const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave), Kp = steps_row(a.K);
    const long m0 = (long)blockIdx.y * (16 * MT);
    const int M = (int)min(a.M - m0, 16L * MT);
    const int n0 = blockIdx.x * 16, row = lane % 16, part = lane / 16;
    const int8_t* w = a.w + (long)min(n0 + row, a.N - 1) * Kp + part * 16;
    auto at = [&](int k, int u) { return k + u * (W * 64); };  // a wave's pieces
    auto in = [&](int k, int u) { return at(k, u) + part * 16 < Kp; };
    i32x4 wv[kFewAhead];
    auto weights = [&](int k) {
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) wv[u] = *reinterpret_cast<const i32x4*>(w + (in(k, u) ? at(k, u) : -part * 16));
    };
    weights(wave * 64);
    if constexpr (kValues) {
        constexpr int kPer = 16 / X::kBytes, kWords = kPer / 4;
        const int slices = W / M, r = wave / slices, slice = wave - r * slices, vecs = a.K / kPer;
        const uint8_t* from = x + (m0 + min(r, M - 1)) * a.x_row * X::kBytes;
        if (t < W) most[t] = 0;
        __syncthreads();
        uint32_t m = 0;
        if (r < M) {
#pragma unroll 4
            for (int c = slice * kWave + lane; c < vecs; c += slices * kWave) m = largest<X>(load16(from + c * 16), m);
            m = lanes_max<kWave>(m);
            if (lane == 0) atomicMax(&most[r], m);
        }
        __syncthreads();
        if (r < M) {
            const Steps st(most[r]);
            if (slice == 0 && lane == 0) scales[r] = st.scale;
#pragma unroll 2
            for (int c = slice * kWave + lane; c * kPer < Kp; c += slices * kWave) {
                uint32_t s[kWords];
                st.of<X>(load16(from + min(c, vecs - 1) * 16), s);
                store_steps<X>(lds + r * Kp + c * kPer, s, c < vecs);
            }
        }
    } else {
        if (t < M) scales[t] = a.x_scale[m0 + t];
    }
    __syncthreads();
    const i32x4 none = {0, 0, 0, 0};
    i32x4 acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = none;
    for (int k = wave * 64; k < Kp;) {
        i32x4 xv[kFewAhead][MT];
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int token = m * 16 + row;
                xv[u][m] = none;
                if (in(k, u) && token < M) {
                    if constexpr (kValues) xv[u][m] = *reinterpret_cast<const i32x4*>(lds + token * Kp + at(k, u) + part * 16);
                    else xv[u][m] = *reinterpret_cast<const i32x4*>(x + (m0 + token) * Kp + at(k, u) + part * 16);
                }
            }
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u], xv[u][m], acc[m], 0, 0, 0);
        k = at(k, kFewAhead);
        if (k < Kp) weights(k);
    }
    if constexpr (kValues) __syncthreads();  // the steps have been read
    // acc[m][r]: channel 4 part + r of token 16 m + row.
    int* sums = reinterpret_cast<int*>(lds);
#pragma unroll
    for (int m = 0; m < MT; ++m) *reinterpret_cast<i32x4*>(sums + wave * (MT * 256) + (m * 16 + row) * 16 + 4 * part) = acc[m];
    __syncthreads();
    static_assert(MT * 4 <= W, "a thread a sum");
    const int n = n0 + t % 16, token = t / 16;
    if (token >= M || n >= a.N) return;
    int s = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) s += sums[i * (MT * 256) + t];
    const float bias = a.bias ? element<T>(a.bias, n) : 0.0f, ws = a.w_scale[n] * kUp;
    store_element<T>(out, (m0 + token) * a.out_row + n, finish<T, ACT>(s, scales[token] * kDown, ws, bias));
}

// Its workgroups.
long few_groups(const Linear8Call& a, int mt) { return (long)((a.N + 15) / 16) * ((a.M + 16 * mt - 1) / (16 * mt)); }

template <class X, class T, int ACT, int MT, int W = 16>
hipError_t few(const Linear8Call& a, const void* x, void* out, hipStream_t st)
{
    constexpr size_t kSums = (size_t)W * MT * 256 * 4;
    const size_t steps = std::is_same<X, Int8>::value ? 0 : (size_t)std::min(a.M, 16L) * steps_row(a.K);
    const auto kernel = few_kernel<X, T, ACT, MT, W>;
    constexpr size_t kMost = std::max(kSums, (size_t)kFewLds) + sizeof(float) * 16 * MT;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), kMost);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
    hipLaunchKernelGGL(kernel, grid, dim3(W * kWave), std::max(kSums, steps), st, a, static_cast<const uint8_t*>(x), out);
    return hipGetLastError();
}

// ---- many tokens -------------------------------------------------------------------------

constexpr int kColumnBytes = 2 << 20;  // weights of a column of tiles: half an L2
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

// Writes NT channels' results of one token from channel i on, those below N, all at once where all are (rows may start at any
// element), past the L2: results that stay there drive out the tokens and weights that the next tiles read (45920 x 4096 x
// 1024, bfloat16: 264 -> 224 us).
template <class T, int NT>
__device__ __forceinline__ void write_channels(uint8_t* to, int i, int N, const float (&v)[NT])
{
    to += (long)i * T::kBytes;
    if constexpr (NT * T::kBytes >= 4) {
        constexpr int kWords = NT * T::kBytes / 4;
        typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
        typedef Words Anywhere __attribute__((aligned(T::kBytes)));
        if (i + NT <= N) {
            Words w;
#pragma unroll
            for (int e = 0; e < kWords; ++e) {
                if constexpr (T::kBytes == 4) {
                    w[e] = __float_as_uint(v[e]);
                } else {
                    typedef float f32x2 __attribute__((ext_vector_type(2)));
                    const f32x2 p = {v[2 * e], v[2 * e + 1]};
                    w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
                }
            }
            __builtin_nontemporal_store(w, reinterpret_cast<Anywhere*>(to));
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < NT; ++e)
        if (i + e < N) store_element<T>(to, e, v[e]);
}

// The order of the tiles: columns of `wide` tiles of channels outside, then tokens, then the column's channels, so that a
// column's weights stay in an L2 while the tokens pass.
struct Order {
    int mtiles, ntiles, wide;
};
struct Tile {
    long m;
    int n;
};
__device__ __forceinline__ Tile tile_at(const Order& o, long i)
{
    const long column = i / ((long)o.mtiles * o.wide), rest = i - column * o.mtiles * o.wide;
    const int first = (int)column * o.wide, width = min(o.wide, o.ntiles - first);
    const long m = rest / width;
    return Tile{m, first + (int)(rest - m * width)};
}

// What a workgroup takes of them: those of its XCD's contiguous share, `slots` workgroups by turns.
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
// one's products run. 45920 x 4096 x 1024 to bfloat16 with GELU 280 us (1380 TOP/s; without it 232), 45888 x 2304 x 768
// 112 (1450). What the first spends without it, in copies with parts left out: products alone 125, with the reads of
// LDS 159, with the loads 202, with the results 232 (a write of their 376 MB alone 55); operands of zeros take 10 to
// 20% less, so power has a share.
template <int BM, int BN, int WM, int WN, int BK, int STAGES, class T, int ACT>
__global__ __launch_bounds__(WM* WN* kWave, 2) void product_kernel(Linear8Call a, const uint8_t* __restrict__ q,
                                                                   const float* __restrict__ q_scale,
                                                                   void* __restrict__ out, Order order)
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
    static_assert(BM <= THREADS, "scales: a thread each");
    extern __shared__ __align__(1024) uint8_t lds[];
    float* scales = reinterpret_cast<float*>(lds + STAGES * kStage);  // [2][BM] of the tokens, by tiles in turns

    const Share sh = share((long)order.mtiles * order.ntiles);
    if (sh.tile >= sh.end) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, half = lane >> 5;
    const int wm = wave % WM, wn = wave / WM;
    const int Kp = steps_row(a.K), chunks = (Kp + BK - 1) / BK, full = Kp / BK;

    // 16 rows of one piece meet the 64 banks once.
    auto swizzle = [](int row) { return kPieces == 8 ? (row >> 1) & 7 : (row >> 2) & 3; };
    // The stream's end that loads: its tile and chunk, and this lane's rows there (load i of a wave brings rows
    // (wave + kWaves i) kRows ... of the buffer), clamped to those that exist.
    const int lrow = lane / kPieces, piece = ((lane % kPieces) ^ swizzle(wave * kRows + lrow)) * 16;
    // Load i is of tokens where its rows lie below BM, uniform over the workgroup; offsets from the tile's first row.
    constexpr int kTokenLoads = BM / kRows / kWaves;
    static_assert(BM % (kRows * kWaves) == 0, "a load is of tokens or of weights");
    uint32_t from[kLoads];
    const uint8_t *qbase = q, *wbase = reinterpret_cast<const uint8_t*>(a.w);
    long ltile = sh.tile;
    int lchunk = 0, lbuf = 0;
    auto place = [&](long tile) {
        const Tile at = tile_at(order, tile);
        const long m0 = at.m * BM;
        const int n0 = at.n * BN;
        qbase = q + m0 * Kp;
        wbase = reinterpret_cast<const uint8_t*>(a.w) + (long)n0 * Kp;
        const int tokens = (int)min((long)BM, a.M - m0) - 1, channels = min(BN, a.N - n0) - 1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = (wave + kWaves * i) * kRows + lrow, c = r - BM;
            // Weight row c of the buffer: row l of fragment f of a wave's NT holds its channel l NT + f, so that a lane's
            // results are NT channels in a row.
            const int channel = c / (32 * NT) * (32 * NT) + c % 32 * NT + c / 32 % NT;
            from[i] = (uint32_t)(i < kTokenLoads ? min(r, tokens) : min(channel, channels)) * (uint32_t)Kp;
        }
    };
    // The values of a tile's channels, a lane's own, and a thread's token's scale on its way to LDS.
    float w_scale[NT], bias[NT], x_scale;
    auto load_scales = [&](long tile) {
        const Tile at = tile_at(order, tile);
        x_scale = q_scale[min(at.m * BM + min(t, BM - 1), a.M - 1)] * kDown;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int c = min(at.n * BN + (wn * 32 + l32) * NT + n, a.N - 1);
            w_scale[n] = a.w_scale[c] * kUp;
            bias[n] = a.bias ? element<T>(a.bias, c) : 0.0f;
        }
    };
    // The loads of the stream's next chunk, one at a time: issued together, they fill the load queue and the products
    // wait behind them. Past the stream's end they go on, over the last tile's chunks, into buffers that nothing reads.
    uint32_t to = 0;
    int at = 0;
    auto aim = [&]() {
        to = (uint32_t)(size_t)(__attribute__((address_space(3))) uint8_t*)(lds + lbuf * kStage + wave * kRows * BK);
        at = min(lchunk * BK + piece, Kp - 16);  // past a row's end the last piece again: the products leave it out
    };
    auto issue = [&](int i) {
        asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(from[i] + at), "s"(i < kTokenLoads ? qbase : wbase),
                     "{m0}"(to + kWaves * i * kRows * BK)
                     : "memory");
    };
    auto issued = [&]() {
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
    // A step of 32 values of k; the loads of a chunk go between the products of its first steps.
    constexpr int kProducts = NT * MT * kSteps32;               // of a chunk
    constexpr int kEvery = kProducts > kLoads ? kProducts / kLoads : 1;
    constexpr int kPer = (kLoads * kEvery + kProducts - 1) / kProducts;  // loads at a time
    auto multiply = [&](int set, int g, bool load) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int p = (g * NT + n) * MT + m;
                if (load && p % kEvery == 0) {
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (p / kEvery * kPer + i < kLoads) issue(p / kEvery * kPer + i);
                }
                acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fx[set][m], fw[set][n], acc[n][m], 0, 0, 0);
            }
    };
    // Chunk c of a tile is there once at most the loads of the kAhead - 1 chunks behind it in the stream are on their
    // way. A tile's first kAhead have been waited for before.
    auto arrive = [&](int c) {
        if (c >= kAhead) wait_loads<kLoads*(kAhead - 1)>();
        lds_barrier();
        aim();
    };

    load_scales(sh.tile);
    place(sh.tile);
    for (int c = 0; c < kAhead; ++c) {
        aim();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) issue(i);
        issued();
    }
    wait_loads<0>();
    int turn = 0;
    auto hand_over = [&]() {  // the scales of the tile that comes
        if (t < BM) scales[turn * BM + t] = x_scale;
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
                multiply(g & 1, g, true);
            }
            issued();
            buf = buf + 1 == STAGES ? 0 : buf + 1;
        }
        if (full < chunks) {
            arrive(full);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) issue(i);
            issued();
            const int left = Kp - full * BK;
#pragma unroll 1
            for (int g = 0; g * 32 < left; ++g) {
                read(0, g);
                if (g * 32 + 16 >= left && half) {  // the second 16 bytes lie past the end
                    const i32x4 none = {0, 0, 0, 0};
#pragma unroll
                    for (int m = 0; m < MT; ++m) fx[0][m] = none;
                }
                multiply(0, 0, false);
            }
            buf = buf + 1 == STAGES ? 0 : buf + 1;
        }

        // Everything on its way has arrived before the first write leaves, so that no wait for loads waits for writes.
        float w[NT], b[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            w[n] = w_scale[n];
            b[n] = bias[n];
        }
        const float* xs = scales + turn * BM + wm * MT * 32 + 4 * half;
        const bool last = tile + sh.slots >= sh.end;
        if (!last) load_scales(tile + sh.slots);
        wait_loads<0>();
        turn ^= 1;
        if (!last) hand_over();
        // acc[n][m][r]: channel l32 NT + n of the wave's, token m * 32 + 8 (r / 4) + 4 half + r % 4. A store writes whole
        // lines of two tokens.
        const Tile place = tile_at(order, tile);
        const long row = place.m * BM + wm * MT * 32 + 4 * half;
        const int at = place.n * BN + (wn * 32 + l32) * NT;
        uint8_t* to = static_cast<uint8_t*>(out) + row * a.out_row * T::kBytes;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(xs + m * 32 + 8 * c);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int token = m * 32 + 8 * c + r;
                    float v[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) v[n] = finish<T, ACT>(acc[n][m][4 * c + r], x[r], w[n], b[n]);
                    if (row + token < a.M)
                        write_channels<T, NT>(to + token * a.out_row * T::kBytes, at, a.N, v);
                }
            }
    }
}

template <int BM, int BN, int WM, int WN, int BK, int STAGES, class T, int ACT>
hipError_t product(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t st)
{
    constexpr size_t bytes = (size_t)STAGES * (BM + BN) * BK + 2 * BM * 4;
    const auto kernel = product_kernel<BM, BN, WM, WN, BK, STAGES, T, ACT>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    const long mtiles = (a.M + BM - 1) / BM, ntiles = (a.N + BN - 1) / BN, per = (mtiles * ntiles + kXcds - 1) / kXcds;
    // As many workgroups as the chip holds (by LDS and by registers: two waves a SIMD).
    constexpr int kHeld = (int)std::min<size_t>((160 << 10) / bytes, 8 / (WM * WN) > 0 ? 8 / (WM * WN) : 1);
    const long slots = std::min(per, (long)kHeld * kUnits / kXcds);
    const int wide = (int)std::max(1L, std::min(ntiles, (long)kColumnBytes / ((long)BN * steps_row(a.K))));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(slots * kXcds)), dim3(WM * WN * kWave), bytes, st, a,
                       reinterpret_cast<const uint8_t*>(q), q_scale, out, Order{(int)mtiles, (int)ntiles, wide});
    return hipGetLastError();
}

// The widest tiles that leave no compute unit idle: a tile of 256 x 256 loads half the bytes a product that one of 128 x 128
// does, which loads half of what one of 64 x 64 does. Tiles of 128 x 256 leave room for two workgroups a compute unit, of
// which one finishes its results beside the other's products: long rows need that least, and there the tiles of 256 x 256,
// one a unit, are taken where they fill half a round of the chip to a whole one, or more than two (between one and two the
// second round is mostly idle). Products (bfloat16 results, no activation), us in tiles of
//                         64    64 x 128    128    128 x 256    256
//     118 x 576 x 192      4.7     5.2      6.9       8.8       9.5
//     4103 x 150 x 848     6.6     7.5     10.4      15.6      18.8
//     1024 x 2304 x 768   10.7     8.0      9.1      11.7      14.1
//     2000 x 1024 x 4096  17.8    15.2     27.4      31.4      47.9
//     7000 x 768 x 3056   46.2    36.8     33.4      35.2      45.9
//     8898 x 1024 x 2528  58.0    55.3     49.3      50.9      40.0
//     45888 x 2304 x 768   200       -      128       112       117
//     45920 x 1024 x 4096  370       -      210       214       182
// Over 90 drawn shapes (32 to 46000 rows, 64 to 5000 channels, 256 to 4096 long) these bounds cost 0.6% against the best of
// the five for each, and 20% at most.
constexpr int kLongRows = 1024;
template <class T, int ACT>
hipError_t product_of(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t st)
{
    // Few tokens or channels: k is split over the waves of a workgroup, where tiles would leave most units idle and walk all
    // of k in each. Such a workgroup has fewer loads on their way than it wants, so the smallest that fill the chip are
    // taken; four token tiles pay for long rows only. Values to results in us, so / in tiles of 64: 63 x 88 x 3968 9.6 / 20.3,
    // 128 x 1024 x 4096 12.3 / 21.6, 250 x 1024 x 4096 16.6 / 21.4, 17 x 2304 x 768 8.3 / 9.4;
    // with four token tiles 1000 x 256 x 256 7.7 / 7.3, 3000 x 64 x 2048 19.4 / 17.9.
    auto groups = [&](int m) { return few_groups(a, m); };
    if (groups(2) <= kUnits || (a.K > 2 * kLongRows && groups(4) <= kUnits)) {
        Linear8Call of = a;
        of.x_scale = q_scale;
        if (groups(1) <= kUnits) return few<Int8, T, ACT, 1>(of, q, out, st);
        if (groups(2) <= kUnits) return few<Int8, T, ACT, 2>(of, q, out, st);
        return few<Int8, T, ACT, 4>(of, q, out, st);
    }
    auto tiles = [&](int m, int n) { return (a.M + m - 1) / m * ((a.N + n - 1) / n); };
    const long area = a.M * (long)a.N / (256 * 256);
    const bool fills = (area >= kUnits / 2 && area <= kUnits) || area >= 2 * kUnits;
    if (a.K > kLongRows && fills) return product<256, 256, 4, 2, 128, 2, T, ACT>(a, q, q_scale, out, st);
    if (tiles(128, 256) >= 2 * kUnits) return product<128, 256, 2, 2, 64, 3, T, ACT>(a, q, q_scale, out, st);
    if (tiles(128, 128) >= kUnits) return product<128, 128, 2, 2, 128, 2, T, ACT>(a, q, q_scale, out, st);
    if (tiles(64, 64) > kUnits) return product<64, 128, 2, 2, 128, 3, T, ACT>(a, q, q_scale, out, st);
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

// Steps made inside the product: a launch less, for tokens that few workgroups read. Replayed without pauses, us, so / by two
// launches: 1 x 2304 x 768 3.9 / 6.3, 100 x 512 x 512 6.2 / 7.9, 4000 x 16 x 256 6.3 / 7.1, 64 x 1024 x 1024 7.6 / 7.5, 8 x 1024 x
// 4096 8.9 / 8.9, 250 x 256 x 2048 11.1 / 8.4, beyond the bound 16 x 4096 x 4096 15.9 / 11.4; called one by one the second
// launch takes 4 us of the host's time besides (250 x 192 x 768 10.5 / 14.5).
bool linear8_is_few(const Linear8Call& a)
{
    return a.x_dt != kI8 && (a.M <= 16 || few_groups(a, 1) <= kUnits) &&
           std::min(a.M, 16L) * steps_row(a.K) <= kFewLds;
}

hipError_t launch_linear8_few(const Linear8Call& a, const void* x, void* out, hipStream_t stream)
{
    return with_kind(a, [&](auto type, auto act) {
        typedef decltype(type) T;
        constexpr int ACT = decltype(act)::value;
        const bool short_rows = a.M <= 4 && steps_row(a.K) <= 4 * kFewAhead * 64;
        auto of = [&](auto x_type) {
            typedef decltype(x_type) X;
            return short_rows ? few<X, T, ACT, 1, 4>(a, x, out, stream) : few<X, T, ACT, 1>(a, x, out, stream);
        };
        return a.x_dt == kBf16 ? of(Bf16{}) : of(F32{});
    });
}

hipError_t launch_linear8(const Linear8Call& a, const int8_t* q, const float* q_scale, void* out, hipStream_t stream)
{
    return with_kind(a, [&](auto type, auto act) {
        return product_of<decltype(type), decltype(act)::value>(a, q, q_scale, out, stream);
    });
}

}  // namespace mpm

// Gradients of the packed attention with a relative position bias, from the stored output and
// softmax statistics (scores and probabilities are recomputed):
//   P = 2^(s - maximum - log2 sum), dP = dO V^T, D_i = dO_i . o_i, dS = P (dP - D),
//   dV = P^T dO, dK = scale dS^T Q, dQ = scale dS K, dbias[offset] = sum of dS over its pairs.
//
// No two workgroups add to one value: a workgroup of the key kernel owns 128 keys and walks the
// queries, one of the query kernel owns 128 queries and walks the keys. That is seven products
// instead of the five of a single pass, for results that are the same on every run.
#include "mpm_attn.h"

namespace mpm {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRowsPerBlock = 32 * kWaves;

template <class S>
constexpr int tile_rows()
{
    return S::kBytes == 2 ? 64 : 32;
}

// D[row][head] = dO . o: eight lanes a (row, head), 16-byte loads.
template <class S>
__global__ __launch_bounds__(kThreads) void delta_kernel(AttentionCall a, HeadRows dout, HeadRows out,
                                                         float* __restrict__ delta)
{
    constexpr int kLanes = 8;
    const int b = blockIdx.y;
    const Rows rq = image_rows(a.q_off, b, a.Nq);
    const long item = ((long)blockIdx.x * kThreads + threadIdx.x) / kLanes;
    const int j = threadIdx.x % kLanes;
    if (item >= (long)rq.count * a.H) return;
    const long row = rq.first + item / a.H;
    const int hd = (int)(item % a.H);
    const uint8_t* x = dout.p + (row * dout.row + (long)hd * dout.head) * S::kBytes;
    const uint8_t* y = out.p + (row * out.row + (long)hd * out.head) * S::kBytes;
    float sum = 0.0f;
    for (int c = j; c * (16 / S::kBytes) < a.dh; c += kLanes) {
        const u32x4 u = load16(x + c * 16), w = load16(y + c * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (S::kBytes == 2) sum += bf16_lo(u[e]) * bf16_lo(w[e]) + bf16_hi(u[e]) * bf16_hi(w[e]);
            else sum += __uint_as_float(u[e]) * __uint_as_float(w[e]);
        }
    }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (j == 0) delta[row * a.H + hd] = sum;
}

// What is taken from a query's scores before the exponential: the maximum and the log of the sum, or
// their sum where it is small enough to hold both (its rounding, below 2^-18, is the error of the
// exponent). A mask value such as -1e9 on every key makes the maximum too large for that: then
// the two go one after the other, as in the forward pass. No key: +inf, so that P = 0.
constexpr float kJoinMost = 64.0f;
struct Taken {
    float first, second;
};
__device__ __forceinline__ bool split_taken(float2 l) { return fabsf(l.x) > kJoinMost && l.x != -__builtin_inff(); }
__device__ __forceinline__ Taken taken(float2 l, bool split)
{
    if (l.x == -__builtin_inff()) return Taken{__builtin_inff(), 0.0f};
    return split ? Taken{l.x, l.y} : Taken{l.x + l.y, 0.0f};
}

// Copies KT rows of two operands into their LDS tiles, zero rows past the end or where dropped.
template <class S, int DH, int ROWS>
__device__ __forceinline__ void stage(uint8_t* ta, uint8_t* tb, const HeadRows& x, const HeadRows& y, long first,
                                      int r0, int count, int head_x, int head_y, int dh, const float* drop, int t)
{
    typedef Tile<S, DH> T;
    for (int e = t; e < ROWS * T::kChunks; e += kThreads) {
        const int r = e / T::kChunks, ch = e % T::kChunks;
        bool in = r0 + r < count;
        if (drop && in) in = drop[first + r0 + r] > -__builtin_inff();
        const long row = first + (in ? r0 + r : 0);
        store16(ta + T::at(r, ch), load_chunk<S>(x.p + (row * x.row + (long)head_x * x.head) * S::kBytes, ch, dh, in));
        store16(tb + T::at(r, ch), load_chunk<S>(y.p + (row * y.row + (long)head_y * y.head) * S::kBytes, ch, dh, in));
    }
}

// dK and dV of 128 keys of one key head: all queries of all heads that share it.
template <class S, int DH, int BIAS>
__global__ __launch_bounds__(kThreads) void key_gradient_kernel(AttentionCall a, HeadRows dout, HeadRows q, HeadRows k,
                                                                HeadRows v, const float2* __restrict__ lse,
                                                                const float* __restrict__ delta, HeadRows dk,
                                                                HeadRows dv, int blocks)
{
    typedef Tile<S, DH> T;
    typedef typename FragOf<S>::type Frag;
    constexpr int QT = tile_rows<S>();
    constexpr int kTileBytes = QT * T::kRowBytes;
    extern __shared__ __align__(16) uint8_t lds[];
    uint8_t* qt = lds;
    uint8_t* ot = lds + kTileBytes;
    int* codes = reinterpret_cast<int*>(lds + 2 * kTileBytes);
    float* lses = reinterpret_cast<float*>(codes + QT);
    float* lows = lses + QT;
    float* deltas = lows + QT;
    int* apart = reinterpret_cast<int*>(deltas + QT);  // whether a query of the tile has its terms taken apart
    float* table = reinterpret_cast<float*>(apart + 4);
    const int table_at = lds_address(table);

    const int pair = blockIdx.x / blocks, blk = blockIdx.x % blocks;
    const int b = pair / a.Hk, hk = pair - b * a.Hk, group = a.H / a.Hk;
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    if (blk * kRowsPerBlock >= rk.count) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, h = lane >> 5;
    const int ki = blk * kRowsPerBlock + wave * 32 + l32;
    const bool exists = ki < rk.count;
    const int W = 2 * a.span + 1;
    const float c = a.scale * kLog2e;
    float kb = exists ? 0.0f : -__builtin_inff();
    if (exists && a.k_bias) kb = to_log2(a.k_bias[rk.first + ki]);
    const bool live = kb > -__builtin_inff();
    const int kcode = bias_code<BIAS>(exists ? (a.k_pos ? a.k_pos[rk.first + ki] : ki) : 0, a.grid_h, a.grid_w, W);

    Frag kf[DH / 16], vf[DH / 16];
    const long krow = rk.first + (exists ? ki : 0);
    load_frags<S, DH>(kf, k.p + (krow * k.row + (long)hk * k.head) * S::kBytes, a.dh, live, h);
    load_frags<S, DH>(vf, v.p + (krow * v.row + (long)hk * v.head) * S::kBytes, a.dh, live, h);

    f32x16 gk[DH / 32], gv[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) gk[d][r] = gv[d][r] = 0.0f;

    for (int hd = hk * group; hd < (hk + 1) * group; ++hd) {
        if (BIAS != kBiasNone) {
            __syncthreads();
            const float* src = a.bias + (long)hd * W * W;
            for (int e = t; e < W * W; e += kThreads) table[e] = to_log2(src[e]);
        }
        for (int q0 = 0; q0 < rq.count; q0 += QT) {
            __syncthreads();
            if (t < QT) {
                const int qi = q0 + t;
                const bool in = qi < rq.count;
                if (BIAS != kBiasNone)
                    codes[t] = query_code<BIAS>(in ? (a.q_pos ? a.q_pos[rq.first + qi] : qi) : 0, a.grid_h, a.grid_w,
                                                a.span, W, table_at);
                const float2 l = in ? lse[(rq.first + qi) * a.H + hd] : make_float2(-__builtin_inff(), 0.0f);
                const bool split = __any(split_taken(l));
                const Taken tk = taken(l, split);
                lses[t] = tk.first;
                lows[t] = tk.second;
                if (t == 0) *apart = split;
                deltas[t] = in ? delta[(rq.first + qi) * a.H + hd] : 0.0f;
            }
            stage<S, DH, QT>(qt, ot, q, dout, rq.first, q0, rq.count, hd, hd, a.dh, nullptr, t);
            __syncthreads();
            const bool split = *apart;
#pragma unroll
            for (int u = 0; u < QT / 32; ++u) {
                f32x16 s, dp;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
                for (int st = 0; st < DH / 16; ++st) {
                    s = mma(rows_frag<S, DH>(qt, 32 * u + l32, st, h), kf[st], s);
                    dp = mma(rows_frag<S, DH>(ot, 32 * u + l32, st, h), vf[st], dp);
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = 32 * u + 8 * g + 4 * h;
                    i32x4 qc = {0, 0, 0, 0};
                    if (BIAS != kBiasNone) qc = *reinterpret_cast<const i32x4*>(codes + at);
                    const f32x4 ls = *reinterpret_cast<const f32x4*>(lses + at);
                    const f32x4 lo = *reinterpret_cast<const f32x4*>(lows + at);
                    const f32x4 de = *reinterpret_cast<const f32x4*>(deltas + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[4 * g + e] * c;
                        if (BIAS != kBiasNone)
                            x = fmaf(s[4 * g + e], c,
                                     lds_at(bias_entry<BIAS>(qc[e], kcode, a.span, W, table_at)));
                        x = x + kb - ls[e];
                        if (split) x -= lo[e];
                        const float p = live ? __builtin_amdgcn_exp2f(x) : 0.0f;
                        s[4 * g + e] = p;
                        dp[4 * g + e] = p * (dp[4 * g + e] - de[e]);
                    }
                }
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const Frag p = tile_frag(s, st, S{}), ds = tile_frag(dp, st, S{});
#pragma unroll
                    for (int d = 0; d < DH / 32; ++d) {
                        gv[d] = mma(cols_frag<S, DH>(ot, 32 * u + 16 * st, 32 * d, lane), p, gv[d]);
                        gk[d] = mma(cols_frag<S, DH>(qt, 32 * u + 16 * st, 32 * d, lane), ds, gk[d]);
                    }
                }
            }
        }
    }

    // A dropped key's gradients are zero, whatever its rows hold.
    if (!live) {
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) gk[d][r] = gv[d][r] = 0.0f;
    }
    store_rows(dk.p + (krow * dk.row + (long)hk * dk.head) * S::kBytes, gk, a.scale, a.dh, exists, h, S{});
    store_rows(dv.p + (krow * dv.row + (long)hk * dv.head) * S::kBytes, gv, 1.0f, a.dh, exists, h, S{});
}

// dQ of 128 queries of one head, and their part of dbias: every dS is added into a table in LDS,
// one wave after the other and the halves of a wave one after the other, so that the order of
// the additions is fixed; the workgroup's table goes to its own slot of `parts`.
template <class S, int DH, int BIAS, bool GRAD>
__global__ __launch_bounds__(kThreads) void query_gradient_kernel(AttentionCall a, HeadRows dout, HeadRows q,
                                                                  HeadRows k, HeadRows v,
                                                                  const float2* __restrict__ lse,
                                                                  const float* __restrict__ delta, HeadRows dq,
                                                                  float* __restrict__ parts, int blocks)
{
    typedef Tile<S, DH> T;
    typedef typename FragOf<S>::type Frag;
    constexpr int KT = tile_rows<S>();
    constexpr int kTileBytes = KT * T::kRowBytes;
    extern __shared__ __align__(16) uint8_t lds[];
    uint8_t* kt = lds;
    uint8_t* vt = lds + kTileBytes;
    int* codes = reinterpret_cast<int*>(lds + 2 * kTileBytes);
    float* kbs = reinterpret_cast<float*>(codes + KT);
    float* table = kbs + KT;
    const int table_at = lds_address(table);

    const int pair = blockIdx.x / blocks, blk = blockIdx.x % blocks;
    const int b = pair / a.H, hd = pair - b * a.H, hk = hd / (a.H / a.Hk);
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    if (blk * kRowsPerBlock >= rq.count) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, h = lane >> 5;
    const int qi = blk * kRowsPerBlock + wave * 32 + l32;
    const bool live = qi < rq.count;
    const int W = 2 * a.span + 1;
    float* sums = table + W * W;
    const float c = a.scale * kLog2e;
    const long qrow = rq.first + (live ? qi : 0);
    const float2 stat = live ? lse[qrow * a.H + hd] : make_float2(-__builtin_inff(), 0.0f);
    const bool split = __any(split_taken(stat));
    const Taken ls = taken(stat, split);
    const float de = live ? delta[qrow * a.H + hd] : 0.0f;

    Frag qf[DH / 16], of[DH / 16];
    load_frags<S, DH>(qf, q.p + (qrow * q.row + (long)hd * q.head) * S::kBytes, a.dh, live, h);
    load_frags<S, DH>(of, dout.p + (qrow * dout.row + (long)hd * dout.head) * S::kBytes, a.dh, live, h);
    int qcode = 0;
    if (BIAS != kBiasNone) {
        qcode = query_code<BIAS>(live ? (a.q_pos ? a.q_pos[qrow] : qi) : 0, a.grid_h, a.grid_w, a.span, W, table_at);
        const float* src = a.bias + (long)hd * W * W;
        for (int e = t; e < W * W; e += kThreads) {
            table[e] = to_log2(src[e]);
            if (GRAD) sums[e] = 0.0f;
        }
    }
    f32x16 gq[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) gq[d][r] = 0.0f;

    for (int k0 = 0; k0 < rk.count; k0 += KT) {
        __syncthreads();
        if (t < KT) {
            const int kk = k0 + t;
            const bool in = kk < rk.count;
            if (BIAS != kBiasNone)
                codes[t] = bias_code<BIAS>(in ? (a.k_pos ? a.k_pos[rk.first + kk] : kk) : 0, a.grid_h, a.grid_w, W);
            kbs[t] = in ? (a.k_bias ? to_log2(a.k_bias[rk.first + kk]) : 0.0f) : -__builtin_inff();
        }
        stage<S, DH, KT>(kt, vt, k, v, rk.first, k0, rk.count, hk, hk, a.dh, a.k_bias, t);
        __syncthreads();
        f32x16 dsum[KT / 32];
#pragma unroll
        for (int u = 0; u < KT / 32; ++u) {
            f32x16 s, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
            for (int st = 0; st < DH / 16; ++st) {
                s = mma(rows_frag<S, DH>(kt, 32 * u + l32, st, h), qf[st], s);
                dp = mma(rows_frag<S, DH>(vt, 32 * u + l32, st, h), of[st], dp);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = 32 * u + 8 * g + 4 * h;
                i32x4 kc = {0, 0, 0, 0};
                if (BIAS != kBiasNone) kc = *reinterpret_cast<const i32x4*>(codes + at);
                const f32x4 kb = *reinterpret_cast<const f32x4*>(kbs + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[4 * g + e] * c;
                    if (BIAS != kBiasNone)
                        x = fmaf(s[4 * g + e], c,
                                 lds_at(bias_entry<BIAS>(qcode, kc[e], a.span, W, table_at)));
                    x = x + kb[e] - ls.first;
                    if (split) x -= ls.second;
                    const float p = kb[e] > -__builtin_inff() ? __builtin_amdgcn_exp2f(x) : 0.0f;
                    dp[4 * g + e] = p * (dp[4 * g + e] - de);
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const Frag ds = tile_frag(dp, st, S{});
#pragma unroll
                for (int d = 0; d < DH / 32; ++d)
                    gq[d] = mma(cols_frag<S, DH>(kt, 32 * u + 16 * st, 32 * d, lane), ds, gq[d]);
            }
            dsum[u] = dp;
        }
        if (GRAD) {
            for (int w = 0; w < 2 * kWaves; ++w) {
                if (wave == w / 2 && h == w % 2 && live) {
#pragma unroll
                    for (int u = 0; u < KT / 32; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int at = 32 * u + 8 * (r / 4) + 4 * h + r % 4;
                            if (k0 + at < rk.count)
                                __hip_atomic_fetch_add(
                                    reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(sums) +
                                                             bias_entry<BIAS>(qcode, codes[at], a.span, W, table_at) - table_at),
                                    dsum[u][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                        }
                }
                __syncthreads();
            }
        }
    }

    if (GRAD) {
        __syncthreads();
        float* part = parts + (long)blockIdx.x * W * W;
        for (int e = t; e < W * W; e += kThreads) part[e] = sums[e];
    }
    store_rows(dq.p + (qrow * dq.row + (long)hd * dq.head) * S::kBytes, gq, a.scale, a.dh, live, h, S{});
}

// dbias[head][e] = the workgroups' parts, images and query blocks in order.
__global__ __launch_bounds__(kThreads) void bias_parts_kernel(AttentionCall a, const float* __restrict__ parts,
                                                              int blocks, float* __restrict__ dbias)
{
    const int W2 = (2 * a.span + 1) * (2 * a.span + 1);
    const int e = blockIdx.x * kThreads + threadIdx.x, hd = blockIdx.y;
    if (e >= W2) return;
    float sum = 0.0f;
    for (int b = 0; b < a.B; ++b) {
        const int n = image_rows(a.q_off, b, a.Nq).count;
        for (int i = 0; i * kRowsPerBlock < n; ++i) sum += parts[(((long)b * a.H + hd) * blocks + i) * W2 + e];
    }
    dbias[(long)hd * W2 + e] = sum;
}

struct Grads {
    HeadRows dq, dk, dv;
    float* delta;
    float* parts;
    float* dbias;
};

int query_blocks(const AttentionCall& a) { return (a.Nq + kRowsPerBlock - 1) / kRowsPerBlock; }

template <class S, int DH, int BIAS>
hipError_t launch_all(const AttentionCall& a, const HeadRows& dout, const HeadRows& q, const HeadRows& k,
                      const HeadRows& v, const HeadRows& out, const float2* lse, const Grads& g, hipStream_t st)
{
    constexpr int R = tile_rows<S>();
    const size_t W2 = (size_t)(2 * a.span + 1) * (2 * a.span + 1);
    const size_t tiles = 2 * R * Tile<S, DH>::kRowBytes, table = BIAS != kBiasNone ? W2 * 4 : 0;
    const long per_image = (long)a.Nq * a.H * 8;
    hipLaunchKernelGGL(delta_kernel<S>, dim3((unsigned)((per_image + kThreads - 1) / kThreads), (unsigned)a.B),
                       dim3(kThreads), 0, st, a, dout, out, g.delta);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    {
        const int blocks = (a.Nk + kRowsPerBlock - 1) / kRowsPerBlock;
        const size_t bytes = tiles + R * 16 + 16 + table;
        const long grid = (long)a.B * a.Hk * blocks;
        if (grid * kThreads > UINT32_MAX) return hipErrorInvalidConfiguration;
        auto kernel = key_gradient_kernel<S, DH, BIAS>;
        if ((e = allow_lds(reinterpret_cast<const void*>(kernel), bytes)) != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), bytes, st, a, dout, q,
                           k, v, lse, g.delta, g.dk, g.dv, blocks);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    const int blocks = query_blocks(a);
    const long grid = (long)a.B * a.H * blocks;
    if (grid * kThreads > UINT32_MAX) return hipErrorInvalidConfiguration;
    const bool grad = BIAS != kBiasNone && g.dbias;
    const size_t bytes = tiles + R * 8 + (grad ? 2 : 1) * table;
    auto kernel = grad ? query_gradient_kernel<S, DH, BIAS, BIAS != kBiasNone>
                       : query_gradient_kernel<S, DH, BIAS, false>;
    if ((e = allow_lds(reinterpret_cast<const void*>(kernel), bytes)) != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), bytes, st, a, dout, q, k, v,
                       lse, g.delta, g.dq, g.parts, blocks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (grad) {
        hipLaunchKernelGGL(bias_parts_kernel, dim3((unsigned)((W2 + kThreads - 1) / kThreads), (unsigned)a.H),
                           dim3(kThreads), 0, st, a, g.parts, blocks, g.dbias);
        e = hipGetLastError();
    }
    return e;
}

template <class S, int DH>
hipError_t pick(const AttentionCall& a, const HeadRows& dout, const HeadRows& q, const HeadRows& k, const HeadRows& v,
                const HeadRows& out, const float2* lse, const Grads& g, hipStream_t st)
{
    switch (bias_kind(a)) {
    case kBiasNone: return launch_all<S, DH, kBiasNone>(a, dout, q, k, v, out, lse, g, st);
    case kBiasGrid: return launch_all<S, DH, kBiasGrid>(a, dout, q, k, v, out, lse, g, st);
    default: return launch_all<S, DH, kBiasFar>(a, dout, q, k, v, out, lse, g, st);
    }
}

size_t aligned256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t attention_backward_bytes(const AttentionCall& a)
{
    const size_t W2 = (size_t)(2 * a.span + 1) * (2 * a.span + 1);
    size_t n = aligned256((size_t)a.B * a.Nq * a.H * 4);
    if (a.bias) n += aligned256((size_t)a.B * a.H * query_blocks(a) * W2 * 4);
    return n;
}

hipError_t launch_attention_backward(const AttentionCall& a, const HeadRows& dout, const HeadRows& q,
                                     const HeadRows& k, const HeadRows& v, const HeadRows& out, const float* lse_pairs,
                                     const HeadRows& dq, const HeadRows& dk, const HeadRows& dv, float* dbias, void* ws,
                                     hipStream_t st)
{
    const float2* lse = reinterpret_cast<const float2*>(lse_pairs);
    float* delta = static_cast<float*>(ws);
    float* parts = reinterpret_cast<float*>(static_cast<char*>(ws) + aligned256((size_t)a.B * a.Nq * a.H * 4));
    const Grads g{dq, dk, dv, delta, parts, dbias};
    if (a.dt == kBf16)
        return a.dh <= 64 ? pick<Bf16, 64>(a, dout, q, k, v, out, lse, g, st)
                          : pick<Bf16, 128>(a, dout, q, k, v, out, lse, g, st);
    return a.dh <= 64 ? pick<F32, 64>(a, dout, q, k, v, out, lse, g, st)
                      : pick<F32, 128>(a, dout, q, k, v, out, lse, g, st);
}

}  // namespace mpm

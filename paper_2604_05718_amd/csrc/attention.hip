// Packed attention with a relative position bias, forward:
//   s_ik = scale q_i . k_k + bias[row_i - row_k][column_i - column_k] + kb_k,
//   o_i = sum_k softmax_k(s)_ik v_k,
// and, for the gradients, the softmax statistics of every query.
//
// One pass over the keys with a running maximum and sum. Scores are kept in base 2 (everything
// is multiplied by log2 e once), so an exponential is one instruction.
#include "mpm_attn.h"

namespace mpm {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kQueriesPerBlock = 32 * kWaves;
constexpr int kXcds = 8;
// The running maximum is raised only when a tile's exceeds it by more than this many powers of
// two: probabilities then stay below 256, exact to scale, and most tiles skip the rescaling.
constexpr float kSlack = 8.0f;

template <class S, int DH>
constexpr int key_tile()
{
    return S::kBytes == 2 ? 64 : 32;
}

// The workgroup's query block and (image, head) pair. Blocks are dealt round-robin to the 8
// XCDs, each with its own L2: pairs are dealt to XCDs whole, so that the blocks that read one
// pair's keys share an L2 (few pairs: in order, since whole pairs would leave XCDs idle).
__device__ __forceinline__ bool block_item(int blocks, int pairs, int* blk, int* pair)
{
    const int i = blockIdx.x;
    if (pairs >= 4 * kXcds) {
        const int slot = i / kXcds;
        *pair = slot / blocks * kXcds + i % kXcds;
        *blk = slot % blocks;
    } else {
        *pair = i / blocks;
        *blk = i % blocks;
    }
    return *pair < pairs;
}

template <class S, int DH, int BIAS, bool KB>
__global__ __launch_bounds__(kThreads) void attention_kernel(AttentionCall a, HeadRows q, HeadRows k, HeadRows v,
                                                             HeadRows out, float* __restrict__ lse, int blocks)
{
    typedef Tile<S, DH> T;
    typedef typename FragOf<S>::type Frag;
    constexpr int KT = key_tile<S, DH>();
    constexpr int kTileBytes = KT * T::kRowBytes;
    extern __shared__ __align__(16) uint8_t lds[];
    uint8_t* kt = lds;
    uint8_t* vt = lds + kTileBytes;
    int* codes = reinterpret_cast<int*>(lds + 2 * kTileBytes);
    float* kbs = reinterpret_cast<float*>(codes + KT);
    float* table = reinterpret_cast<float*>(kbs + KT);

    int blk, pair;
    if (!block_item(blocks, a.B * a.H, &blk, &pair)) return;
    const int b = pair / a.H, hd = pair - b * a.H, hk = hd / (a.H / a.Hk);
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    if (blk * kQueriesPerBlock >= rq.count) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, h = lane >> 5;
    const int qi = blk * kQueriesPerBlock + wave * 32 + l32;
    const bool live = qi < rq.count;
    const int W = 2 * a.span + 1;
    const float c = a.scale * kLog2e;

    Frag qf[DH / 16];
    const uint8_t* qrow = q.p + ((rq.first + (live ? qi : 0)) * q.row + (long)hd * q.head) * S::kBytes;
    load_frags<S, DH>(qf, qrow, a.dh, live, h);
    int qcode = 0;
    if (BIAS != kBiasNone) {
        qcode = query_code<BIAS>(live ? (a.q_pos ? a.q_pos[rq.first + qi] : qi) : 0, a.grid_h, a.grid_w, a.span, W);
        const float* src = a.bias + (long)hd * W * W;
        for (int e = t; e < W * W; e += kThreads) table[e] = to_log2(src[e]);
    }

    f32x16 acc[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.0f;
    float m = -__builtin_inff(), sum = 0.0f;

    for (int k0 = 0; k0 < rk.count; k0 += KT) {
        __syncthreads();
        if (t < KT) {
            const int kk = k0 + t;
            const bool in = kk < rk.count;
            if (BIAS != kBiasNone)
                codes[t] = bias_code<BIAS>(in ? (a.k_pos ? a.k_pos[rk.first + kk] : kk) : 0, a.grid_h, a.grid_w, W);
            if (KB) kbs[t] = in ? to_log2(a.k_bias[rk.first + kk]) : -__builtin_inff();
        }
        for (int e = t; e < KT * T::kChunks; e += kThreads) {
            const int r = e / T::kChunks, ch = e % T::kChunks, kk = k0 + r;
            bool in = kk < rk.count;
            if (KB && in) in = a.k_bias[rk.first + kk] > -__builtin_inff();  // a dropped key's rows are not read
            const long row = rk.first + (in ? kk : 0);
            store16(kt + T::at(r, ch), load_chunk<S>(k.p + (row * k.row + (long)hk * k.head) * S::kBytes, ch, a.dh, in));
            store16(vt + T::at(r, ch), load_chunk<S>(v.p + (row * v.row + (long)hk * v.head) * S::kBytes, ch, a.dh, in));
        }
        __syncthreads();

        f32x16 s[KT / 32];
#pragma unroll
        for (int u = 0; u < KT / 32; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[u][r] = 0.0f;
#pragma unroll
            for (int st = 0; st < DH / 16; ++st) s[u] = mma(rows_frag<S, DH>(kt, 32 * u + l32, st, h), qf[st], s[u]);
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < KT / 32; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = 32 * u + 8 * g + 4 * h;
                i32x4 kc = {0, 0, 0, 0};
                f32x4 kb = {0, 0, 0, 0};
                if (BIAS != kBiasNone) kc = *reinterpret_cast<const i32x4*>(codes + at);
                if (KB) kb = *reinterpret_cast<const f32x4*>(kbs + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[u][4 * g + e];
                    if (BIAS != kBiasNone) {
                        const int en = bias_entry<BIAS>(qcode, kc[e], a.span, W);
                        x = fmaf(x, c, *reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(table) + en));
                    } else {
                        x *= c;
                    }
                    if (KB) x = kb[e] > -__builtin_inff() ? x + kb[e] : -__builtin_inff();
                    else if (k0 + KT > rk.count) x = k0 + at + e < rk.count ? x : -__builtin_inff();
                    s[u][4 * g + e] = x;
                    top = fmaxf(top, x);
                }
            }
        top = halves_max(top);
        if (__any(top > m + kSlack)) {
            const float up = fmaxf(m, top);
            const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - up);
            m = up;
            sum *= f;
#pragma unroll
            for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= f;
        }
        const float base = m == -__builtin_inff() ? 0.0f : m;  // every key so far masked
#pragma unroll
        for (int u = 0; u < KT / 32; ++u) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[u][r] = __builtin_amdgcn_exp2f(s[u][r] - base);
                sum += s[u][r];
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const Frag p = tile_frag(s[u], st, S{});
#pragma unroll
                for (int d = 0; d < DH / 32; ++d)
                    acc[d] = mma(cols_frag<S, DH>(vt, 32 * u + 16 * st, 32 * d, lane), p, acc[d]);
            }
        }
    }

    sum = halves_sum(sum);
    if (!live) return;
    const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);  // no key: zeros
    uint8_t* orow = out.p + ((rq.first + qi) * out.row + (long)hd * out.head) * S::kBytes;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = 32 * d + 8 * g + 4 * h;
            if (at < a.dh)
                store4(orow + at * S::kBytes, acc[d][4 * g] * inv, acc[d][4 * g + 1] * inv, acc[d][4 * g + 2] * inv,
                       acc[d][4 * g + 3] * inv, S{});
        }
    if (lse && h == 0)
        reinterpret_cast<float2*>(lse)[(rq.first + qi) * a.H + hd] =
            sum == 0.0f ? make_float2(-__builtin_inff(), 0.0f) : make_float2(m, __builtin_log2f(sum));
}

template <class S, int DH, int BIAS, bool KB>
hipError_t launch(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v, const HeadRows& out,
                  float* lse, hipStream_t stream)
{
    constexpr int KT = key_tile<S, DH>();
    const int W = 2 * a.span + 1;
    const size_t bytes = 2 * KT * Tile<S, DH>::kRowBytes + KT * 8 + (BIAS != kBiasNone ? (size_t)W * W * 4 : 0);
    const int blocks = (a.Nq + kQueriesPerBlock - 1) / kQueriesPerBlock;
    const long pairs = (long)a.B * a.H;
    const long grid = (pairs >= 4 * kXcds ? (pairs + kXcds - 1) / kXcds * kXcds : pairs) * blocks;
    if (grid * kThreads > UINT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = attention_kernel<S, DH, BIAS, KB>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), bytes, stream, a, q, k, v, out, lse, blocks);
    return hipGetLastError();
}

template <class S, int DH>
hipError_t pick(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v, const HeadRows& out,
                float* lse, hipStream_t st)
{
    const int bias = bias_kind(a);
    if (a.k_bias) {
        if (bias == kBiasNone) return launch<S, DH, kBiasNone, true>(a, q, k, v, out, lse, st);
        if (bias == kBiasGrid) return launch<S, DH, kBiasGrid, true>(a, q, k, v, out, lse, st);
        return launch<S, DH, kBiasFar, true>(a, q, k, v, out, lse, st);
    }
    if (bias == kBiasNone) return launch<S, DH, kBiasNone, false>(a, q, k, v, out, lse, st);
    if (bias == kBiasGrid) return launch<S, DH, kBiasGrid, false>(a, q, k, v, out, lse, st);
    return launch<S, DH, kBiasFar, false>(a, q, k, v, out, lse, st);
}

}  // namespace

hipError_t launch_attention(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v,
                            const HeadRows& out, float* lse, hipStream_t st)
{
    if (a.dt == kBf16)
        return a.dh <= 64 ? pick<Bf16, 64>(a, q, k, v, out, lse, st) : pick<Bf16, 128>(a, q, k, v, out, lse, st);
    return a.dh <= 64 ? pick<F32, 64>(a, q, k, v, out, lse, st) : pick<F32, 128>(a, q, k, v, out, lse, st);
}

}  // namespace mpm

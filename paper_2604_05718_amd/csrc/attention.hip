// Packed attention with a relative position bias, forward:
//   s_ik = scale q_i . k_k + bias[row_i - row_k][column_i - column_k] + kb_k,
//   o_i = sum_k softmax_k(s)_ik v_k,
// and, for the gradients, the softmax statistics of every query.
//
// One pass over the keys with a running maximum and sum. Scores are kept in base 2 (everything
// is multiplied by log2 e once), so an exponential is one instruction.
//
// Bound by instruction issue: a score costs an exponential, its share of a bias read, a maximum, a sum and
// a conversion, and those and the products hardly overlap (3 images of 4096 tokens: vector instructions
// 49% and products 26% of the busy cycles), as a wave finishes 32 keys before it starts the next 32. A score
// tile's registers are the next product's operand, so scores never pass through LDS; one barrier a key tile.
// Bfloat16, heads of 64: 8 images of 4096 tokens, 16 heads, 712 us, 770 TFLOP/s (a product of 8192 reaches 1227);
// 64 of about 717, 12 heads, 222 us, 460 TFLOP/s (a sixth of a workgroup's time is its first loads and its last
// stores); float32, 5 images of about 590, 6 heads of 40, 60 us. (After some 30 calls in a row: in the first
// 20 ms of work the card is up to a third slower.)
//
// Heads of 72 to 128 channels keep part of their fragments in scratch memory, 24 to 108 bytes a lane in bfloat16
// and 316 to 448 in float32; of the others six do, 8 to 32 bytes.
#include "mpm_attn.h"

namespace mpm {
namespace {

// What is taken from a query's scores (base 2) before the exponential need not be their maximum: floats
// keep their precision at any scale. It is zero as long as the scores stay within this many powers of two
// of it, so that most calls subtract nothing, and else follows the running maximum with that slack.
// The slack comes out of the range of the values: the sums of 2^14 keys hold values up to 2^(128 - 14 - 16),
// and the terms of weight 2^-24 beside the largest are normal numbers for values from 2^(16 + 24 - 126).
constexpr float kSlack = 16.0f;

template <class S, int SPLIT>
constexpr int key_tile()
{
    return S::kBytes == 2 ? 64 : 32 * SPLIT;
}

// One of the two buffers: a tile of keys and of values, their position codes and biases.
template <class S, int DH, int SPLIT>
constexpr int buffer_bytes()
{
    return key_tile<S, SPLIT>() * (2 * Tile<S, DH>::kRowBytes + 8);
}

// Waves a SIMD the registers are held to: three of 32 queries (64 channels, bfloat16; 168 registers and
// 250 us, 64 images of about 717 tokens, against 170 and 295 us with two), two elsewhere.
template <class S, int DH, int QT>
constexpr int waves_per_simd()
{
    return S::kBytes == 2 && DH == 64 && QT == 1 ? 3 : 2;
}

// WAVES waves of QT tiles of 32 queries each share the key tiles. SPLIT 2: two waves share 32 queries,
// each taking every other 32 keys, and join their maxima, sums and outputs at the end. STATS: with the sum of the
// unrounded probabilities for the statistics (float32: the only sum). Bfloat16 divides by the sum of the rounded ones
// (frag_sum): the unrounded sum for both / this, without statistics 64 images of about 717 tokens 244 / 253 us, 8 of
// 4096 750 / 752; with both sums there a step of 3 images of 4096 tokens takes 2% more. One kernel with both sums 255
// and 804.
template <class S, int DH, int BIAS, bool KB, int WAVES, int QT, int SPLIT, bool STATS>
__global__ __launch_bounds__(WAVES* kWave, (waves_per_simd<S, DH, QT>())) void attention_kernel(AttentionCall a, HeadRows q, HeadRows k, HeadRows v,
                                                                HeadRows out, float* __restrict__ lse, int blocks)
{
    constexpr int THREADS = WAVES * kWave;
    static_assert(SPLIT == 1 || (SPLIT == 2 && QT == 1), "a split tile is one tile");
    constexpr int KT = key_tile<S, SPLIT>();
    typedef PairStage<S, DH, KT, THREADS, true> Staged;
    typedef typename FragOf<S>::type Frag;
    constexpr int kBuffer = buffer_bytes<S, DH, SPLIT>();
    constexpr bool kBf = S::kBytes == 2;
    extern __shared__ __align__(16) uint8_t lds[];
    float* table = reinterpret_cast<float*>(lds + 2 * kBuffer);
    const int table_at = lds_address(table);

    int blk, pair;
    if (!block_item(blocks, a.B * a.H, &blk, &pair)) return;
    const int b = pair / a.H, hd = pair - b * a.H, hk = hd / (a.H / a.Hk);
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    const int q0 = blk * (32 * WAVES * QT / SPLIT);
    if (q0 >= rq.count) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave / SPLIT, l32 = lane & 31, h = lane >> 5;
    const int part = t / kWave % SPLIT;
    const int W = 2 * a.span + 1;
    const float c = a.scale * kLog2e;

    Staged stage;
    int pos = 0;
    float kbias = 0.0f;
    const float* drop = KB ? a.k_bias + rk.first : nullptr;
    auto load = [&](int k0) {
        stage.template load<KB>(a.dh, rk.count, drop, k0, t);
        if (t < KT) {
            const int kk = k0 + t;
            const bool in = kk < rk.count;
            if (BIAS != kBiasNone) pos = in ? (a.k_pos ? a.k_pos[rk.first + kk] : kk) : 0;
            if (KB) kbias = in ? drop[kk] : -__builtin_inff();
        }
    };
    auto store = [&](int buf) {
        uint8_t* at = lds + buf * kBuffer;
        stage.template store<KB>(at, t);
        if (t < KT) {
            int* codes = reinterpret_cast<int*>(at + 2 * Staged::kTileBytes);
            if (BIAS != kBiasNone) codes[t] = bias_code<BIAS>(pos, a.grid_h, a.grid_w, W);
            if (KB) reinterpret_cast<float*>(codes + KT)[t] = to_log2(kbias);
        }
    };
    stage.init(k, v, rk.first, hk, a.dh, t);
    load(0);

    Frag qf[QT][DH / 16];
    int qcode[QT];
    f32x16 acc[QT][DH / 32];
    float m[QT], sum[QT], used[QT];  // what is taken from the scores; the sums: unrounded, and (bfloat16) rounded
    bool fresh[QT];        // no key yet
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int qi = q0 + (wave * QT + i) * 32 + l32;
        const bool live = qi < rq.count;
        load_frags<S, DH>(qf[i], q.p + ((rq.first + (live ? qi : 0)) * q.row + (long)hd * q.head) * S::kBytes, a.dh, live,
                          h);
        // (the position for now: the first loads are all under way before one is waited for)
        qcode[i] = BIAS != kBiasNone && live ? (a.q_pos ? a.q_pos[rq.first + qi] : qi) : 0;
        m[i] = sum[i] = used[i] = 0.0f;
        fresh[i] = true;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][d][r] = 0.0f;
    }
    if (BIAS != kBiasNone) {
        load_table<THREADS>(table, a.bias + (long)hd * W * W, W * W, t);
#pragma unroll
        for (int i = 0; i < QT; ++i)
            qcode[i] = query_code<BIAS>(qcode[i], a.grid_h, a.grid_w, a.span, W, table_at);
    }
    store(0);
    __syncthreads();

    const bool works = q0 + wave * QT * 32 < rq.count;  // a wave past the image's end only brings tiles
    bool shifted = false, any_fresh = true;  // whether a query of the wave has m != 0, or no key yet
    for (int k0 = 0, buf = 0; k0 < rk.count; k0 += KT, buf ^= 1) {
        const uint8_t* kt = lds + buf * kBuffer;
        const uint8_t* vt = kt + Staged::kTileBytes;
        const int* codes = reinterpret_cast<const int*>(vt + Staged::kTileBytes);
        const float* kbs = reinterpret_cast<const float*>(codes + KT);
        const bool more = k0 + KT < rk.count;
        if (more) load(k0 + KT);
        auto compute = [&](int u) {
            f32x16 s[QT];
#pragma unroll
            for (int st = 0; st < DH / 16; ++st) {
                if (!kBf && st > 0 && 16 * st >= a.dh) continue;  // (a float32 step is worth a branch)
                const Frag kf = rows_frag<S, DH>(kt, 32 * u + l32, st, h);
                const f32x16 zero = {};
#pragma unroll
                for (int i = 0; i < QT; ++i) s[i] = mma(kf, qf[i][st], st == 0 ? zero : s[i]);
            }
            bool up_any = any_fresh;
            float top[QT];
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                top[i] = -__builtin_inff();
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = 32 * u + 8 * g + 4 * h;
                    i32x4 kc = {0, 0, 0, 0};
                    f32x4 kb = {0, 0, 0, 0};
                    if (BIAS != kBiasNone) kc = *reinterpret_cast<const i32x4*>(codes + at);
                    if (KB) kb = *reinterpret_cast<const f32x4*>(kbs + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[i][4 * g + e];
                        if (BIAS != kBiasNone) {
                            x = fmaf(x, c, lds_at(bias_entry<BIAS>(qcode[i], kc[e], a.span, W, table_at)));
                        } else {
                            x *= c;
                        }
                        if (KB) x = kb[e] == -__builtin_inff() ? kb[e] : x + kb[e];
                        s[i][4 * g + e] = x;
                    }
                }
                if (!KB && k0 + 32 * u + 32 > rk.count) {
                    int left = rk.count - k0 - 32 * u - 4 * h;
                    asm volatile("" : "+v"(left));  // keeps this a branch: no selects in whole tiles
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r / 4) + r % 4 >= left) s[i][r] = -__builtin_inff();
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) top[i] = fmaxf(top[i], s[i][r]);
                up_any |= top[i] > m[i] + kSlack;
            }
            if (__any(up_any)) {
                shifted = any_fresh = false;
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    const float full = halves_max(top[i]);
                    float to = m[i];
                    const bool first = fresh[i];
                    if (first) {
                        // A first key: zero does for scores that are neither large nor all very small.
                        if (full > -__builtin_inff()) {
                            to = fabsf(full) <= kSlack ? 0.0f : full;
                            fresh[i] = false;
                        }
                    } else if (full > m[i] + kSlack) {
                        to = full;
                    }
                    const float f = first ? 0.0f : __builtin_amdgcn_exp2f(m[i] - to);
                    m[i] = to;
                    if (STATS) sum[i] *= f;
                    if (kBf) used[i] *= f;
#pragma unroll
                    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][d][r] *= f;
                    shifted |= __any(to != 0.0f);
                    any_fresh |= __any(fresh[i]);
                }
            }
            if (shifted) {
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    float by = m[i];
                    asm volatile("" : "+v"(by));  // keeps this a branch
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[i][r] -= by;
                }
            }
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[i][r] = __builtin_amdgcn_exp2f(s[i][r]);
                    if (STATS) sum[i] += s[i][r];
                }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                Frag p[QT];
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    p[i] = tile_frag(s[i], st, S{});
                    used[i] = frag_sum(p[i], used[i]);
                }
#pragma unroll
                for (int d = 0; d < DH / 32; ++d) {
                    if (!kBf && d > 0 && 32 * d >= a.dh) continue;
                    const Frag vf = cols_frag<S, DH>(vt, 32 * u + 16 * st, 32 * d, lane);
#pragma unroll
                    for (int i = 0; i < QT; ++i) acc[i][d] = mma(vf, p[i], acc[i][d]);
                }
            }
        };
        if (works) {
            if constexpr (SPLIT == 1) {
                // Unrolled for constant LDS offsets; one tile's registers at a time.
#pragma unroll
                for (int u = 0; u < KT / 32; ++u) {
                    compute(u);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                for (int u = part; u < KT / 32; u += SPLIT) compute(u);
            }
        }
        if (more) store(buf ^ 1);
        __syncthreads();
    }

    if constexpr (SPLIT == 2) {
        constexpr int kPad = DH + 4;  // floats of a query's outputs, apart in banks
        float* mine = reinterpret_cast<float*>(lds) + (wave * 32 + l32) * kPad;
        float4* stats = reinterpret_cast<float4*>(reinterpret_cast<float*>(lds) + WAVES / 2 * 32 * kPad) + wave * kWave + lane;
        static_assert((WAVES / 2 * 32 * kPad + WAVES / 2 * kWave * 4) * 4 <= 2 * kBuffer, "the joined outputs fit");
        if (part == 1) {
            *stats = make_float4(fresh[0] ? -__builtin_inff() : m[0], sum[0], used[0], 0.0f);
#pragma unroll
            for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<float4*>(mine + 32 * d + 8 * g + 4 * h) =
                        make_float4(acc[0][d][4 * g], acc[0][d][4 * g + 1], acc[0][d][4 * g + 2], acc[0][d][4 * g + 3]);
        }
        __syncthreads();
        if (part == 1) return;
        const float4 other = *stats;
        const float own = fresh[0] ? -__builtin_inff() : m[0], top = fmaxf(own, other.x);
        const float f = fresh[0] ? 0.0f : __builtin_amdgcn_exp2f(own - top);
        const float o = other.x == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(other.x - top);
        m[0] = top;
        if (STATS) sum[0] = f * sum[0] + o * other.y;
        if (kBf) used[0] = f * used[0] + o * other.z;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(mine + 32 * d + 8 * g + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[0][d][4 * g + e] = f * acc[0][d][4 * g + e] + o * x[e];
            }
    }
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        const int qi = q0 + (wave * QT + i) * 32 + l32;
        const float by = halves_sum(kBf ? used[i] : sum[i]);
        const bool live = qi < rq.count;
        const float inv = by > 0.0f ? 1.0f / by : (by == 0.0f ? 0.0f : by);  // no key: zeros
        store_rows(out.p + ((rq.first + (live ? qi : 0)) * out.row + (long)hd * out.head) * S::kBytes, acc[i], inv, a.dh,
                   live, h, S{});
        if constexpr (STATS) {
            const float total = halves_sum(sum[i]);
            if (lse && live && h == 0)
                reinterpret_cast<float2*>(lse)[(rq.first + qi) * a.H + hd] =
                    total == 0.0f ? make_float2(-__builtin_inff(), 0.0f) : make_float2(m[i], __builtin_log2f(total));
        }
    }
}

template <class S, int DH, int BIAS, bool KB, int WAVES, int QT, int SPLIT>
hipError_t launch_as(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v,
                     const HeadRows& out, float* lse, hipStream_t stream)
{
    constexpr int THREADS = WAVES * kWave, kQueries = 32 * WAVES * QT / SPLIT;
    const int W = 2 * a.span + 1;
    const size_t bytes = 2 * buffer_bytes<S, DH, SPLIT>() + (BIAS != kBiasNone ? (size_t)W * W * 4 : 0);
    const int blocks = (a.Nq + kQueries - 1) / kQueries;
    const long grid = block_grid((long)a.B * a.H, blocks);
    if (grid * THREADS > UINT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = attention_kernel<S, DH, BIAS, KB, WAVES, QT, SPLIT, true>;
    if constexpr (S::kBytes == 2)
        if (lse == nullptr) kernel = attention_kernel<S, DH, BIAS, KB, WAVES, QT, SPLIT, false>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(THREADS), bytes, stream, a, q, k, v, out, lse, blocks);
    return hipGetLastError();
}

// (Heads of up to 64 channels; wider ones have the form of four waves alone.)
// Eight waves of 64 queries where an image has queries for several such blocks, or where the bias
// table leaves LDS for one workgroup only; otherwise four waves of 32, three workgroups a compute
// unit. Bfloat16, 64 channels, 12 heads, four waves / eight: 8 images of 4096 tokens without a bias
// 527 / 484 us, with one of 127 x 127 (16 heads) 1810 / 770, 8 of 2304 with one of 95 x 95 288 / 236, 8 of
// about 1380 144 / 149, 64 of about 717 with one of 63 x 63 254 / 287, one of 1024 41 / 60.
// Two waves share 32 queries where workgroups of 128 would be few (not split / split): bfloat16, 12 heads of
// up to 1024 tokens, 72 workgroups 35 / 28 us, 288 42 / 37, 576 48 / 56, 1152 79 / 88; float32, 6 heads of
// up to 576, 96 workgroups 71 / 49, 384 100 / 106, 768 174 / 173.
template <class S, int DH, int BIAS, bool KB>
hipError_t launch(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v, const HeadRows& out,
                  float* lse, hipStream_t stream)
{
    constexpr long kLargeTable = 48 << 10;
    constexpr long kFewGroups = 384;
    if constexpr (S::kBytes == 2 && DH == 64) {
        const long W = 2 * a.span + 1;
        const bool one = BIAS != kBiasNone && W * W * 4 > kLargeTable;  // one workgroup a compute unit
        if (a.Nq >= 1792 || (BIAS != kBiasNone && W * W * 4 > kLargeTable && a.Nq > 256))
        {
            // Rounds over the compute units, in units of the 512-query workgroup's time: one of 256 queries
            // takes 0.6 of it (8 images of 4096 tokens, 16 heads: 918 us against 770 in full rounds; 3
            // images, 768 workgroups against 384, 360 against 408).
            const long pairs = (long)a.B * a.H;
            const long wide = (pairs * ((a.Nq + 511) / 512) + 255) / 256, narrow = (pairs * ((a.Nq + 255) / 256) + 255) / 256;
            if constexpr (BIAS != kBiasNone)
                if (one && 0.6 * (double)narrow < (double)wide)
                    return launch_as<S, DH, BIAS, KB, 8, 1, 1>(a, q, k, v, out, lse, stream);
            return launch_as<S, DH, BIAS, KB, 8, 2, 1>(a, q, k, v, out, lse, stream);
        }
    }
    if constexpr (DH == 64) {
        const long groups = (long)a.B * a.H * ((a.Nq + 127) / 128);
        if (groups < kFewGroups && a.Nk > 32) return launch_as<S, DH, BIAS, KB, 4, 1, 2>(a, q, k, v, out, lse, stream);
    }
    return launch_as<S, DH, BIAS, KB, 4, 1, 1>(a, q, k, v, out, lse, stream);
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

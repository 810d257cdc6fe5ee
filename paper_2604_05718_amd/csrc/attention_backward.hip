// Gradients of the packed attention with a relative position bias, from the stored output and
// softmax statistics (scores and probabilities are recomputed):
//   P = 2^(s - maximum - log2 sum), dP = dO V^T, D_i = dO_i . o_i, dS = P (dP - D),
//   dV = P^T dO, dK = scale dS^T Q, dQ = scale dS K, dbias[offset] = sum of dS over its pairs.
//
// No two workgroups add to one value: a workgroup of the key kernel owns its keys and walks the
// queries, one of the query kernel owns its queries and walks the keys. That is seven products
// instead of the five of a single pass, for results that are the same on every run.
//
// dbias is a histogram: every score gradient belongs to the offset of its pair. Each workgroup of
// the query kernel keeps a table of all offsets in LDS and adds to it with 64-bit integer atomics, whose
// sum does not depend on their order. The unit is a power of two for which no sum can pass the integer's
// range, found from the largest |dS|, which the key kernel, running first, leaves for every image and head:
// at most 2^-39 of it (256 queries and 16384 keys; 2^-44 for 128 and 1024), so that far offsets under sharp
// attention keep their gradients. (32 bits cost 2% less of a step of 32 images of about 717 tokens, 9% less of one
// of 3 of 4096 with 127 x 127 entries, and lose every term below 2^-23 of the largest.)
#include "mpm_attn.h"

namespace mpm {
namespace {

constexpr int kDeltaThreads = 256;

// How the query kernel sums dbias.
enum SumKind : int {
    kSumNone = 0,
    kSumBeside = 1,  // biases and sums in LDS
    // Tables too wide for both (more than 103 x 103 entries): the sums in LDS, the biases read from memory, on
    // their way during a tile's products. A step of 3 images of 4096 tokens, 16 heads of 64, bfloat16: 1.46 ms
    // with 127 x 127 entries, 1.99 with 111 x 111 (offsets held to the span).
    kSumAlone = 2
};

template <class S, int DH, int SPLIT>
constexpr int tile_rows()
{
    return S::kBytes == 2 && DH == 64 ? 64 : 32 * SPLIT;
}
// Buffers of row tiles in LDS: two, or one where two would not leave room for the tables.
template <class S, int DH>
constexpr int buffers()
{
    return S::kBytes == 4 && DH == 128 ? 1 : 2;
}
template <class S, int DH, int SPLIT>
constexpr int tile_bytes()
{
    return 2 * tile_rows<S, DH, SPLIT>() * Tile<S, DH>::kRowBytes;
}

// A split wave's sums join its partner's through LDS: N tiles a lane, in tile order.
template <int N>
__device__ __forceinline__ void give(float* lds, const f32x16 (&x)[N], int lane)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *reinterpret_cast<float4*>(lds + ((n * 4 + r / 4) * kWave + lane) * 4) =
                make_float4(x[n][r], x[n][r + 1], x[n][r + 2], x[n][r + 3]);
}
template <int N>
__device__ __forceinline__ void take(const float* lds, f32x16 (&x)[N], int lane)
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(lds + ((n * 4 + r / 4) * kWave + lane) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][r + e] += v[e];
        }
}

// Waves a SIMD the registers are held to: float32 fragments take twice the registers (a step of 4
// images of about 460 tokens: 275 us with two waves, in scratch memory, 205 with one).
template <class S>
constexpr int waves_per_simd()
{
    return S::kBytes == 2 ? 2 : 1;
}

// What the kernels leave for each other: D of every query and head, the largest |dS| of every image and head
// (as bits). D is kept by image slot, not by packed row: the packed offsets of a call on some images of a larger
// tensor start past zero.
struct Scratch {
    float* delta;       // [B][Nq][H]
    uint32_t* largest;  // [B][H]
    float* parts;       // [pair][block][W * W]
};

// D[row][head] = dO . o: eight lanes a (row, head), 16-byte loads. Also clears the words that the
// key kernel collects in. Bound by memory: 32 images of about 717 rows of 768, bfloat16, 71 MB in 13 us.
//
// In bfloat16 the output carries its own rounding and that of the probabilities, and so does D: an error
// of one sign along a query's row of dS. It is lost among the other roundings in dq, dk, dv and dbias,
// and shows where few buckets sum many offsets, whose terms cancel: 5 x 5 buckets over 9 x 9 to 127 x 127 offsets,
// images of 25 to 4096 tokens, the table's gradient differs from 64 bits by 0.0020 to 0.0037 of its norm, 0.0015 to
// 0.0019 in float32 rounded at the end; a bucket an offset: 0.0017 both. D from unrounded probabilities would take a
// pass of two more products over all pairs.
template <class S>
__global__ __launch_bounds__(kDeltaThreads) void delta_kernel(AttentionCall a, HeadRows dout, HeadRows out, Scratch w)
{
    constexpr int kLanes = 8;
    const int b = blockIdx.y;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.H; i += kDeltaThreads) w.largest[(long)b * a.H + i] = 0;
    const Rows rq = image_rows(a.q_off, b, a.Nq);
    const long item = ((long)blockIdx.x * kDeltaThreads + threadIdx.x) / kLanes;
    const int j = threadIdx.x % kLanes;
    if (item >= (long)rq.count * a.H) return;
    const long row = rq.first + item / a.H;
    const int hd = (int)(item % a.H);  // (item: also the entry in this image's slots)
    const uint8_t* x = dout.p + (row * dout.row + (long)hd * dout.head) * S::kBytes;
    const uint8_t* y = out.p + (row * out.row + (long)hd * out.head) * S::kBytes;
    float sum = 0.0f;
    for (int c = j; c * (16 / S::kBytes) < a.dh; c += kLanes) {
        const u32x4 u = load16(x + c * 16), v = load16(y + c * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (S::kBytes == 2) sum += bf16_lo(u[e]) * bf16_lo(v[e]) + bf16_hi(u[e]) * bf16_hi(v[e]);
            else sum += __uint_as_float(u[e]) * __uint_as_float(v[e]);
        }
    }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (j == 0) w.delta[(long)b * a.Nq * a.H + item] = sum;
}

// What is taken from a query's scores before the exponential: the maximum and the log of the sum
// (`apart`), or their sum where it is small enough to hold both (the log is at most 16, the forward's slack, and
// 14 for the keys: the sum stays below 128 and its rounding, the error of the exponent, below 2^-18). A mask
// value such as -1e9 on every key makes the maximum too large for that: then the two go one after the other, as
// in the forward pass. In bfloat16 calls the sum is not subtracted at all: the score products start from minus
// it over the factor of the scores.
constexpr float kJoinMost = 64.0f;
__device__ __forceinline__ bool too_large(float2 l) { return fabsf(l.x) > kJoinMost && l.x > -__builtin_inff(); }

template <class S>
__device__ __forceinline__ bool can_start(float c)
{
    return S::kBytes == 2 && c > 1e-3f && c < 1e3f;
}

// Two numbers for a query with statistics l: (where the score products start, 0), or, apart, what is
// subtracted first and second. No key: probabilities of zero.
__device__ __forceinline__ float2 taken(float2 l, bool apart, float c)
{
    const bool none = l.x == -__builtin_inff();
    if (apart) return none ? make_float2(__builtin_inff(), 0.0f) : l;
    return make_float2(none ? -__builtin_inff() : -(l.x + l.y) / c, 0.0f);
}

// dK and dV of WAVES x 32 keys of one key head: all queries of all heads that share it. SPLIT 2 (here and
// below): two waves share 32 rows, each taking every other 32 of the other side, and add up at the end.
// Four products a tile, of which two read their operand transposed from LDS. 3 images of 4096 tokens,
// 16 heads of 64, bfloat16: 514 us, 800 TFLOP/s; 32 of about 717, 12 heads: 181 us. Products 34% of the
// busy cycles, vector instructions 48%, LDS 16%, and a wave waits 40% of its time: two waves a SIMD are what
// the fragments and two gradient tiles of a wave leave room for. Heads of 72 to 128 channels pass them, with 300
// to 444 bytes a lane in scratch memory (float32, at one wave a SIMD: 36 to 92).
template <class S, int DH, int BIAS, bool KB, int WAVES, int SPLIT>
__global__ __launch_bounds__(WAVES* kWave, (waves_per_simd<S>())) void key_gradient_kernel(AttentionCall a, HeadRows dout, HeadRows q,
                                                                      HeadRows k, HeadRows v,
                                                                      const float2* __restrict__ lse, Scratch w,
                                                                      HeadRows dk, HeadRows dv, int blocks)
{
    constexpr int THREADS = WAVES * kWave, QT = tile_rows<S, DH, SPLIT>(), BUFS = buffers<S, DH>();
    typedef PairStage<S, DH, QT, THREADS, false> Staged;
    typedef typename FragOf<S>::type Frag;
    constexpr int kBuffer = tile_bytes<S, DH, SPLIT>() + QT * 16 + 16;
    extern __shared__ __align__(16) uint8_t lds[];
    float* table = reinterpret_cast<float*>(lds + BUFS * kBuffer);
    const int table_at = lds_address(table);

    int blk, pair;
    if (!block_item(blocks, (long)a.B * a.Hk, &blk, &pair)) return;
    const int b = pair / a.Hk, hk = pair - b * a.Hk, group = a.H / a.Hk;
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    const int k0 = blk * (32 * WAVES / SPLIT);
    if (k0 >= rk.count) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave / SPLIT, l32 = lane & 31, h = lane >> 5;
    const int share = t / kWave % SPLIT;
    const int ki = k0 + wave * 32 + l32;
    const bool exists = ki < rk.count;
    const bool works = k0 + wave * 32 < rk.count;  // a wave past the image's end only brings tiles
    const int W = 2 * a.span + 1;
    const float c = a.scale * kLog2e;
    const bool start = can_start<S>(c);
    float kb = 0.0f;
    if (KB) kb = exists ? to_log2(a.k_bias[rk.first + ki]) : -__builtin_inff();
    int kcode = 0;
    const bool live = exists && kb != -__builtin_inff();
    // (all of the first loads are under way before one is waited for)
    int own = 0;  // this key's position
    if (BIAS != kBiasNone) own = exists ? (a.k_pos ? a.k_pos[rk.first + ki] : ki) : 0;

    Frag kf[DH / 16], vf[DH / 16];
    const long krow = rk.first + (exists ? ki : 0);
    load_frags<S, DH>(kf, k.p + (krow * k.row + (long)hk * k.head) * S::kBytes, a.dh, live, h);
    load_frags<S, DH>(vf, v.p + (krow * v.row + (long)hk * v.head) * S::kBytes, a.dh, live, h);

    f32x16 gk[DH / 32], gv[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) gk[d][r] = gv[d][r] = 0.0f;

    Staged stage;
    int pos = 0;
    float2 stat;
    float del = 0.0f;
    for (int hd = hk * group; hd < (hk + 1) * group; ++hd) {
        auto load = [&](int q0) {
            stage.template load<false>(a.dh, rq.count, nullptr, q0, t);
            if (t < QT) {
                const int qi = q0 + t;
                const bool in = qi < rq.count;
                // (past the image's end: the last query's, so that only entries that a pair has are read)
                const int at = min(qi, rq.count - 1);
                if (BIAS != kBiasNone) pos = at < 0 ? 0 : a.q_pos ? a.q_pos[rq.first + at] : at;
                stat = in ? lse[(rq.first + qi) * a.H + hd] : make_float2(-__builtin_inff(), 0.0f);
                del = in ? w.delta[((long)b * a.Nq + qi) * a.H + hd] : 0.0f;
            }
        };
        auto store = [&](int buf) {
            uint8_t* at = lds + buf * kBuffer;
            stage.template store<false>(at, t);
            if (t < QT) {  // one wave (or half of one)
                int* codes = reinterpret_cast<int*>(at + tile_bytes<S, DH, SPLIT>());
                float* first = reinterpret_cast<float*>(codes + QT);
                if (BIAS != kBiasNone) codes[t] = query_code<BIAS>(pos, a.grid_h, a.grid_w, a.span, W, table_at);
                const bool apart = !start || __any(too_large(stat));
                const float2 tk = taken(stat, apart, c);
                first[t] = tk.x;
                first[QT + t] = tk.y;
                first[2 * QT + t] = -del;
                if (t == 0) reinterpret_cast<int*>(first + 3 * QT)[0] = apart;
            }
        };
        __syncthreads();
        stage.init(q, dout, rq.first, hd, a.dh, t);
        load(0);
        if (BIAS != kBiasNone) {
            load_table<THREADS>(table, a.bias + (long)hd * W * W, W * W, t);
            kcode = bias_code<BIAS>(own, a.grid_h, a.grid_w, W);
        }
        store(0);
        __syncthreads();
        float most = 0.0f;
        for (int q0 = 0, buf = 0; q0 < rq.count; q0 += QT, buf ^= BUFS - 1) {
            const uint8_t* qt = lds + buf * kBuffer;
            const uint8_t* ot = qt + Staged::kTileBytes;
            const int* codes = reinterpret_cast<const int*>(ot + Staged::kTileBytes);
            const float* first = reinterpret_cast<const float*>(codes + QT);
            const bool more = q0 + QT < rq.count;
            if (more) load(q0 + QT);
            const bool apart = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int*>(first + 3 * QT)[0]);
            auto compute = [&](int u) {
                f32x16 s, dp;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = 32 * u + 8 * g + 4 * h;
                    f32x4 x = {0, 0, 0, 0};
                    if (!apart) x = *reinterpret_cast<const f32x4*>(first + at);
                    const f32x4 y = *reinterpret_cast<const f32x4*>(first + 2 * QT + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[4 * g + e] = x[e];
                        dp[4 * g + e] = y[e];
                    }
                }
#pragma unroll
                for (int st = 0; st < DH / 16; ++st) {
                    if (S::kBytes == 4 && 16 * st >= a.dh) continue;  // (a float32 step is worth a branch)
                    s = mma(rows_frag<S, DH>(qt, 32 * u + l32, st, h), kf[st], s);
                    dp = mma(rows_frag<S, DH>(ot, 32 * u + l32, st, h), vf[st], dp);
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    i32x4 qc = {0, 0, 0, 0};
                    if (BIAS != kBiasNone) qc = *reinterpret_cast<const i32x4*>(codes + 32 * u + 8 * g + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[4 * g + e];
                        if (BIAS != kBiasNone) x = fmaf(x, c, lds_at(bias_entry<BIAS>(qc[e], kcode, a.span, W, table_at)));
                        else x *= c;
                        if (KB) x += kb;
                        s[4 * g + e] = x;
                    }
                }
                if (apart) {
                    const float* from = first;
                    asm volatile("" : "+v"(from));  // keeps this a branch
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int at = 32 * u + 8 * (r / 4) + 4 * h + r % 4;
                        s[r] = s[r] - from[at] - from[QT + at];
                    }
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = __builtin_amdgcn_exp2f(s[r]);
                    dp[r] *= s[r];
                    if (BIAS != kBiasNone) most = fmaxf(most, fabsf(dp[r]));
                }
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const Frag p = tile_frag(s, st, S{}), ds = tile_frag(dp, st, S{});
#pragma unroll
                    for (int d = 0; d < DH / 32; ++d) {
                        if (S::kBytes == 4 && 32 * d >= a.dh) continue;
                        gv[d] = mma(cols_frag<S, DH>(ot, 32 * u + 16 * st, 32 * d, lane), p, gv[d]);
                        gk[d] = mma(cols_frag<S, DH>(qt, 32 * u + 16 * st, 32 * d, lane), ds, gk[d]);
                    }
                }
            };
            if (works) {
#pragma unroll 1
                for (int u = share; u < QT / 32; u += SPLIT) compute(u);
            }
            if (BUFS == 1) __syncthreads();
            if (more) store(buf ^ (BUFS - 1));
            __syncthreads();
        }
        if (BIAS != kBiasNone) {
            if (!live) most = 0.0f;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
            if (lane == 0)
                __hip_atomic_fetch_max(w.largest + (long)b * a.H + hd, __float_as_uint(most), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
        }
    }

    if constexpr (SPLIT == 2) {
        float* mine = reinterpret_cast<float*>(lds) + wave * (2 * DH / 32 * 16 * kWave);
        static_assert(WAVES / 2 * 2 * DH / 32 * 16 * kWave * 4 <= BUFS * kBuffer, "the shared sums fit");
        if (share == 1) {
            give(mine, gk, lane);
            give(mine + DH / 32 * 16 * kWave, gv, lane);
        }
        __syncthreads();
        if (share == 1) return;
        take(mine, gk, lane);
        take(mine + DH / 32 * 16 * kWave, gv, lane);
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

// Largest power of two lg for which x 2^lg < 2^bits (zero and what is not finite: any).
__device__ __forceinline__ int raise_to(float x, int bits)
{
    if (!(x > 0.0f) || !(x < __builtin_inff())) return 0;
    return bits - __builtin_amdgcn_frexp_expf(x);
}
// Bits of a term, so that `terms` of them stay within 62 (and one within the 51 that a double's fixed point holds).
__device__ __forceinline__ int term_bits(int terms) { return min(50, 62 - (32 - __builtin_clz(max(terms - 1, 1)))); }

// Bytes of the query kernel's tables.
__host__ __device__ constexpr size_t table_bytes(int bias, int sum, int W)
{
    if (bias == kBiasNone) return 0;
    return (size_t)W * W * (sum == kSumNone ? 4 : sum == kSumBeside ? 12 : 8);
}

// dQ of WAVES x 32 queries of one head, and their part of dbias. Tables in LDS: the biases and then the sums
// (the sums first; kSumAlone: the sums only). Three products a tile, and an LDS atomic a score: 3 images of 4096
// tokens, 16 heads of 64, bfloat16, 574 us, 540 TFLOP/s (biases from memory); 32 of about 717, 12 heads, 201 us;
// float32, 4 of about 460, 6 heads, 69 us. Vector instructions 64% of the busy cycles, products 22%, LDS 18%.
// Bfloat16 heads of 72 to 128 channels keep 84 to 288 bytes a lane in scratch memory.
template <class S, int DH, int BIAS, bool KB, int SUM, int WAVES, int SPLIT>
__global__ __launch_bounds__(WAVES* kWave, (waves_per_simd<S>())) void query_gradient_kernel(AttentionCall a, HeadRows dout, HeadRows q,
                                                                        HeadRows k, HeadRows v,
                                                                        const float2* __restrict__ lse, Scratch w,
                                                                        HeadRows dq, int blocks)
{
    constexpr int THREADS = WAVES * kWave, KT = tile_rows<S, DH, SPLIT>(), BUFS = buffers<S, DH>();
    typedef PairStage<S, DH, KT, THREADS, true> Staged;
    typedef typename FragOf<S>::type Frag;
    typedef __attribute__((address_space(3))) unsigned long long lds_long;
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    constexpr int kBuffer = tile_bytes<S, DH, SPLIT>() + KT * 8;
    extern __shared__ __align__(16) uint8_t lds[];
    const int W = 2 * a.span + 1, W2 = W * W;
    unsigned long long* sums = reinterpret_cast<unsigned long long*>(lds + BUFS * kBuffer);
    float* table = reinterpret_cast<float*>(sums + (SUM == kSumNone ? 0 : W2));
    const int table_at = SUM == kSumAlone ? 0 : lds_address(table), sums_at = lds_address(sums) - 2 * table_at;

    int blk, pair;
    if (!block_item(blocks, (long)a.B * a.H, &blk, &pair)) return;
    const int b = pair / a.H, hd = pair - b * a.H, hk = hd / (a.H / a.Hk);
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    const int q0 = blk * (32 * WAVES / SPLIT);
    if (q0 >= rq.count) return;
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave / SPLIT, l32 = lane & 31, h = lane >> 5;
    const int share = t / kWave % SPLIT;
    const int qi = q0 + wave * 32 + l32;
    const bool live = qi < rq.count;
    const bool works = q0 + wave * 32 < rq.count;  // a wave past the image's end only brings tiles
    const float c = a.scale * kLog2e;
    const long qrow = rq.first + (live ? qi : 0);

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
            int* codes = reinterpret_cast<int*>(at + tile_bytes<S, DH, SPLIT>());
            if (BIAS != kBiasNone) codes[t] = bias_code<BIAS>(pos, a.grid_h, a.grid_w, W);
            if (KB) reinterpret_cast<float*>(codes + KT)[t] = to_log2(kbias);
        }
    };
    stage.init(k, v, rk.first, hk, a.dh, t);
    load(0);
    const int qat = min(qi, rq.count - 1);  // (past the image's end: the last query's, as in the key kernel)
    const int qpos = BIAS != kBiasNone ? (a.q_pos ? a.q_pos[rq.first + qat] : qat) : 0;
    Frag qf[DH / 16], of[DH / 16];
    load_frags<S, DH>(qf, q.p + (qrow * q.row + (long)hd * q.head) * S::kBytes, a.dh, live, h);
    load_frags<S, DH>(of, dout.p + (qrow * dout.row + (long)hd * dout.head) * S::kBytes, a.dh, live, h);

    // Score gradients in fixed point: added to 1.5 x 2^(52 - lg), a double's bits count units of 2^-lg.
    int lg = 0;
    if (SUM != kSumNone)
        lg = __builtin_amdgcn_readfirstlane(raise_to(__uint_as_float(w.largest[(long)b * a.H + hd]),
                                                     term_bits(32 * WAVES / SPLIT * rk.count)));
    const double middle = __builtin_ldexp(1.5, 52 - lg);
    const float2 stat = live ? lse[qrow * a.H + hd] : make_float2(-__builtin_inff(), 0.0f);
    const bool apart = !can_start<S>(c) || __any(too_large(stat));
    const float2 tk = taken(stat, apart, c);
    const float nd = live ? -w.delta[((long)b * a.Nq + qi) * a.H + hd] : 0.0f;
    f32x16 s0, dp0;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s0[r] = apart ? 0.0f : tk.x;
        dp0[r] = nd;
    }
    int qcode = 0;
    const float* bias = BIAS != kBiasNone ? a.bias + (long)hd * W2 : nullptr;
    if (BIAS != kBiasNone) {
        if (SUM != kSumAlone) load_table<THREADS>(table, bias, W2, t);
        qcode = query_code<BIAS>(qpos, a.grid_h, a.grid_w, a.span, W, table_at);
        if (SUM != kSumNone)
            for (int e = t; e < W2; e += THREADS) sums[e] = 0;
    }
    f32x16 gq[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) gq[d][r] = 0.0f;
    store(0);
    __syncthreads();

    for (int k0 = 0, buf = 0; k0 < rk.count; k0 += KT, buf ^= BUFS - 1) {
        const uint8_t* kt = lds + buf * kBuffer;
        const uint8_t* vt = kt + Staged::kTileBytes;
        const int* codes = reinterpret_cast<const int*>(vt + Staged::kTileBytes);
        const float* kbs = reinterpret_cast<const float*>(codes + KT);
        const bool more = k0 + KT < rk.count;
        if (more) load(k0 + KT);
        auto compute = [&](int u) {
            f32x16 s, dp;
            int entry[16];
            float beside[16];  // kSumAlone: the biases, on their way during the products
            auto find = [&]() {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const i32x4 kc = *reinterpret_cast<const i32x4*>(codes + 32 * u + 8 * g + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at = bias_entry<BIAS>(qcode, kc[e], a.span, W, table_at);
                        entry[4 * g + e] = at;
                        if (SUM == kSumAlone)
                            beside[4 * g + e] = *reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(bias) + at);
                    }
                }
            };
            if constexpr (SUM == kSumAlone) find();
#pragma unroll
            for (int st = 0; st < DH / 16; ++st) {
                if (S::kBytes == 4 && st > 0 && 16 * st >= a.dh) continue;
                s = mma(rows_frag<S, DH>(kt, 32 * u + l32, st, h), qf[st], st == 0 ? s0 : s);
                dp = mma(rows_frag<S, DH>(vt, 32 * u + l32, st, h), of[st], st == 0 ? dp0 : dp);
            }
            if constexpr (BIAS != kBiasNone && SUM != kSumAlone) find();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                f32x4 kb = {0, 0, 0, 0};
                if (KB) kb = *reinterpret_cast<const f32x4*>(kbs + 32 * u + 8 * g + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[4 * g + e];
                    if (BIAS == kBiasNone) x *= c;
                    else if (SUM == kSumAlone) x = fmaf(x, c, to_log2(beside[4 * g + e]));
                    else x = fmaf(x, c, lds_at(entry[4 * g + e]));
                    if (KB) x = kb[e] == -__builtin_inff() ? kb[e] : x + kb[e];
                    s[4 * g + e] = x;
                }
            }
            if (!KB && k0 + 32 * u + 32 > rk.count) {
                int left = rk.count - k0 - 32 * u - 4 * h;
                asm volatile("" : "+v"(left));  // keeps this a branch: no selects in whole tiles
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (8 * (r / 4) + r % 4 >= left) s[r] = -__builtin_inff();
            }
            if (apart) {
                float one = tk.x;
                asm volatile("" : "+v"(one));
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = s[r] - one - tk.y;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] *= __builtin_amdgcn_exp2f(s[r]);
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const Frag ds = tile_frag(dp, st, S{});
#pragma unroll
                for (int d = 0; d < DH / 32; ++d)
                    if (S::kBytes == 2 || 32 * d < a.dh) gq[d] = mma(cols_frag<S, DH>(kt, 32 * u + 16 * st, 32 * d, lane), ds, gq[d]);
            }
            if (SUM != kSumNone) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const u32x2 d = __builtin_bit_cast(u32x2, (double)dp[r] + middle);
                    const u32x2 n = {d[0], d[1] - (uint32_t)__double2hiint(middle)};  // (middle's low word is zero)
                    __hip_atomic_fetch_add((lds_long*)(uintptr_t)(uint32_t)(entry[r] * 2 + sums_at),
                                           __builtin_bit_cast(unsigned long long, n), __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_WORKGROUP);
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
                for (int u = share; u < KT / 32; u += SPLIT) compute(u);
            }
        }
        if (BUFS == 1) __syncthreads();
        if (more) store(buf ^ (BUFS - 1));
        __syncthreads();
    }

    const double back = __builtin_ldexp(1.0, -lg);
    if constexpr (SPLIT == 2) {
        float* mine = reinterpret_cast<float*>(lds) + wave * (DH / 32 * 16 * kWave);
        static_assert(WAVES / 2 * DH / 32 * 16 * kWave * 4 <= BUFS * kBuffer, "the shared sums fit");
        if (share == 1) give(mine, gq, lane);
        __syncthreads();
        if (share == 0) take(mine, gq, lane);
    }
    if (SUM != kSumNone) {
        // A gradient that is not a number is not one in the sums either: it has reached dq.
        bool bad = false;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) bad |= !(fabsf(gq[d][r]) < __builtin_inff());
        const bool any_bad = __syncthreads_or(bad && live && share == 0);
        float* part = w.parts + ((long)pair * blocks + blk) * W2;
        for (int e = t; e < W2; e += THREADS)
            part[e] = any_bad ? __builtin_nanf("") : (float)((double)(long long)sums[e] * back);
    }
    store_rows(dq.p + (qrow * dq.row + (long)hd * dq.head) * S::kBytes, gq, a.scale, a.dh, live && share == 0, h, S{});
}

// dbias[head][e] = the workgroups' parts, in the order of images and query blocks: four threads an
// entry take every fourth image, joined in order.
constexpr int kJoinEntries = 64, kJoinWays = 4;
__global__ __launch_bounds__(kJoinEntries* kJoinWays) void bias_parts_kernel(AttentionCall a,
                                                                           const float* __restrict__ parts, int blocks,
                                                                           int rows, float* __restrict__ dbias)
{
    __shared__ float joined[kJoinWays][kJoinEntries];
    const int W2 = (2 * a.span + 1) * (2 * a.span + 1);
    const int col = threadIdx.x % kJoinEntries, way = threadIdx.x / kJoinEntries, hd = blockIdx.y;
    const int e = min((int)blockIdx.x * kJoinEntries + col, W2 - 1);
    float sum = 0.0f;
    for (int b = way; b < a.B; b += kJoinWays) {
        const int n = (image_rows(a.q_off, b, a.Nq).count + rows - 1) / rows;
        const float* part = parts + ((long)b * a.H + hd) * blocks * W2 + e;
#pragma unroll 4
        for (int i = 0; i < n; ++i) sum += part[(long)i * W2];
    }
    joined[way][col] = sum;
    __syncthreads();
    if (way != 0 || (int)blockIdx.x * kJoinEntries + col >= W2) return;
#pragma unroll
    for (int x = 1; x < kJoinWays; ++x) sum += joined[x][col];
    dbias[(long)hd * W2 + e] = sum;
}

struct Grads {
    HeadRows dq, dk, dv;
    float* dbias;
    Scratch w;
};

struct Inputs {
    HeadRows dout, q, k, v, out;
    const float2* lse;
};

// Eight waves where the query kernel's tables (12 bytes an entry beside 33 KB of tiles) leave LDS for one
// workgroup only. A step, four waves / eight: 32 images of about 717 tokens with 63 x 63 entries, the widest for two
// workgroups, 567 / 609 us; 24 of about 760 with 65 x 65 644 / 533, of about 910 with 71 x 71 789 / 678.
constexpr int kWidestTwice = 63;
bool large_table(const AttentionCall& a) { return a.dt == kBf16 && a.dh <= 64 && a.bias && 2 * a.span + 1 > kWidestTwice; }
// Waves of a workgroup and how many share a tile: split where workgroups of 128 rows would leave
// compute units idle (and the tables of a float32 call leave room for the longer tiles). Heads of up to 64
// channels; wider ones are not split. A whole step, not split / split: bfloat16, 12 heads of 1024 tokens, 96
// workgroups 131 / 112 us, 192 142 / 134, 288 162 / 190, 576 259 / 269; float32, 6 heads of 576 tokens, 90
// workgroups 247 / 182, 180 271 / 303, 360 479 / 447, 720 731 / 823 (by how the rounds over the compute units end).
struct Shape {
    int waves, split;
    int rows() const { return 32 * waves / split; }
};
constexpr long kFewGroups = 256;
constexpr size_t kLdsBytes = 160 << 10;
Shape shape(const AttentionCall& a)
{
    if (large_table(a)) return Shape{8, 1};
    const long groups = (long)a.B * a.H * ((a.Nq + 127) / 128), W = 2 * a.span + 1;
    const bool room = a.dt == kBf16 || !a.bias || W * W * 12 + (66L << 10) <= (long)kLdsBytes;
    return Shape{4, a.dh <= 64 && groups < kFewGroups && room ? 2 : 1};
}
int block_rows(const AttentionCall& a) { return shape(a).rows(); }
int query_blocks(const AttentionCall& a) { return (a.Nq + block_rows(a) - 1) / block_rows(a); }

template <class S, int DH, int BIAS, bool KB, int WAVES, int SPLIT>
hipError_t launch_keys(const AttentionCall& a, const Inputs& in, const Grads& g, hipStream_t st)
{
    const size_t W = 2 * a.span + 1;
    constexpr int kRows = 32 * WAVES / SPLIT;
    const int blocks = (a.Nk + kRows - 1) / kRows;
    const size_t bytes = buffers<S, DH>() * (tile_bytes<S, DH, SPLIT>() + tile_rows<S, DH, SPLIT>() * 16 + 16) +
                         (BIAS != kBiasNone ? W * W * 4 : 0);
    const long grid = block_grid((long)a.B * a.Hk, blocks);
    if (grid * WAVES * kWave > UINT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = key_gradient_kernel<S, DH, BIAS, KB, WAVES, SPLIT>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(WAVES * kWave), bytes, st, a, in.dout, in.q, in.k, in.v,
                       in.lse, g.w, g.dk, g.dv, blocks);
    return hipGetLastError();
}

template <class S, int DH, int BIAS, bool KB, int SUM, int WAVES, int SPLIT>
hipError_t launch_queries(const AttentionCall& a, const Inputs& in, const Grads& g, hipStream_t st)
{
    const int blocks = query_blocks(a);
    const size_t bytes = buffers<S, DH>() * (tile_bytes<S, DH, SPLIT>() + tile_rows<S, DH, SPLIT>() * 8) +
                         table_bytes(BIAS, SUM, 2 * a.span + 1);
    const long grid = block_grid((long)a.B * a.H, blocks);
    if (grid * WAVES * kWave > UINT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = query_gradient_kernel<S, DH, BIAS, KB, SUM, WAVES, SPLIT>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(WAVES * kWave), bytes, st, a, in.dout, in.q, in.k, in.v,
                       in.lse, g.w, g.dq, blocks);
    return hipGetLastError();
}

template <class S, int DH, int BIAS, bool KB, int WAVES, int SPLIT>
hipError_t launch_all(const AttentionCall& a, const Inputs& in, const Grads& g, hipStream_t st)
{
    const int W = 2 * a.span + 1;
    const long per_image = (long)a.Nq * a.H * 8;
    hipLaunchKernelGGL(delta_kernel<S>, dim3((unsigned)((per_image + kDeltaThreads - 1) / kDeltaThreads), (unsigned)a.B),
                       dim3(kDeltaThreads), 0, st, a, in.dout, in.out, g.w);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = launch_keys<S, DH, BIAS, KB, WAVES, SPLIT>(a, in, g, st);
    if (e != hipSuccess) return e;
    if constexpr (BIAS == kBiasNone) {
        return launch_queries<S, DH, BIAS, KB, kSumNone, WAVES, SPLIT>(a, in, g, st);
    } else {
        constexpr size_t tiles = buffers<S, DH>() * (tile_bytes<S, DH, SPLIT>() + tile_rows<S, DH, SPLIT>() * 8);
        if (!g.dbias) return launch_queries<S, DH, BIAS, KB, kSumNone, WAVES, SPLIT>(a, in, g, st);
        // (shape() takes the forms that kSumAlone is not built for where both tables fit only)
        constexpr bool wide = SPLIT == 1 && (S::kBytes == 4 || DH == 128 || WAVES == 8);
        if (!wide || tiles + table_bytes(BIAS, kSumBeside, W) <= kLdsBytes) {
            e = launch_queries<S, DH, BIAS, KB, kSumBeside, WAVES, SPLIT>(a, in, g, st);
        } else {
            if constexpr (wide) e = launch_queries<S, DH, BIAS, KB, kSumAlone, WAVES, SPLIT>(a, in, g, st);
        }
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(bias_parts_kernel, dim3((unsigned)((W * W + kJoinEntries - 1) / kJoinEntries), (unsigned)a.H),
                           dim3(kJoinEntries * kJoinWays), 0, st, a, g.w.parts, query_blocks(a), 32 * WAVES / SPLIT, g.dbias);
        return hipGetLastError();
    }
}

template <class S, int DH, int BIAS, int WAVES, int SPLIT>
hipError_t pick_drop(const AttentionCall& a, const Inputs& in, const Grads& g, hipStream_t st)
{
    return a.k_bias ? launch_all<S, DH, BIAS, true, WAVES, SPLIT>(a, in, g, st)
                    : launch_all<S, DH, BIAS, false, WAVES, SPLIT>(a, in, g, st);
}

template <class S, int DH, int BIAS>
hipError_t pick_shape(const AttentionCall& a, const Inputs& in, const Grads& g, hipStream_t st)
{
    const Shape s = shape(a);
    if constexpr (S::kBytes == 2 && DH == 64 && BIAS != kBiasNone)
        if (s.waves == 8) return pick_drop<S, DH, BIAS, 8, 1>(a, in, g, st);
    if constexpr (DH == 64)
        if (s.split == 2) return pick_drop<S, DH, BIAS, 4, 2>(a, in, g, st);
    return pick_drop<S, DH, BIAS, 4, 1>(a, in, g, st);
}

template <class S, int DH>
hipError_t pick(const AttentionCall& a, const Inputs& in, const Grads& g, hipStream_t st)
{
    switch (bias_kind(a)) {
    case kBiasNone: return pick_shape<S, DH, kBiasNone>(a, in, g, st);
    case kBiasGrid: return pick_shape<S, DH, kBiasGrid>(a, in, g, st);
    default: return pick_shape<S, DH, kBiasFar>(a, in, g, st);
    }
}

size_t aligned256(size_t v) { return (v + 255) / 256 * 256; }

// The scratch regions' sizes, in order (the last one for dbias only, so that a call without it has the others
// where they are).
struct Sizes {
    size_t delta, largest, parts;
};
Sizes sizes(const AttentionCall& a)
{
    const size_t W = 2 * a.span + 1;
    return Sizes{aligned256((size_t)a.B * a.Nq * a.H * 4), aligned256((size_t)a.B * a.H * 4),
                 a.bias ? aligned256((size_t)a.B * a.H * query_blocks(a) * W * W * 4) : 0};
}

}  // namespace

size_t attention_backward_bytes(const AttentionCall& a, bool with_dbias)
{
    const Sizes n = sizes(a);
    return n.delta + n.largest + (with_dbias ? n.parts : 0);
}

hipError_t launch_attention_backward(const AttentionCall& a, const HeadRows& dout, const HeadRows& q,
                                     const HeadRows& k, const HeadRows& v, const HeadRows& out, const float* lse,
                                     const HeadRows& dq, const HeadRows& dk, const HeadRows& dv, float* dbias, void* ws,
                                     hipStream_t st)
{
    const Sizes n = sizes(a);
    char* p = static_cast<char*>(ws);
    const Scratch w{reinterpret_cast<float*>(p), reinterpret_cast<uint32_t*>(p + n.delta),
                    reinterpret_cast<float*>(p + n.delta + n.largest)};
    const Inputs in{dout, q, k, v, out, reinterpret_cast<const float2*>(lse)};
    const Grads g{dq, dk, dv, dbias, w};
    if (a.dt == kBf16) return a.dh <= 64 ? pick<Bf16, 64>(a, in, g, st) : pick<Bf16, 128>(a, in, g, st);
    return a.dh <= 64 ? pick<F32, 64>(a, in, g, st) : pick<F32, 128>(a, in, g, st);
}

}  // namespace mpm

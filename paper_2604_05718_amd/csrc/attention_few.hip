// Attention of a few queries over many keys: the queries of all heads that share a key head are the
// 32 columns of one tile (mpm_attn.h), and the keys are split, over the four waves of a workgroup
// and over workgroups, whose running maxima, sums and unscaled outputs are joined afterwards.
//
// Bound by memory: every key and value is read once. A wave keeps its own tile of 32 values in LDS
// and the next tile's keys, values and bias entries in registers on their way, so waves never wait
// for each other; with one live column in 32 the products cost less than the bytes. Bias entries are
// read from memory (a table in LDS would cost more to bring than the few columns read of it), their
// keys' positions a tile earlier still: entries asked for only when needed made every tile wait for
// its successor's loads (82 -> 72 us). One query an image over 16384 keys, 4 images of 16 heads of 64,
// bfloat16: 268 MB in 53 us (5.0 TB/s), and 6 us to join the splits. Float32 heads of 72 to 128 channels keep
// 630 to 870 bytes a lane in scratch memory, bfloat16 ones with a bias and float32 ones of up to 64 with a key bias
// 56 to 104.
#include <algorithm>

#include "mpm_attn.h"

namespace mpm {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kCols = 32;
constexpr float kSlack = 8.0f;  // scores may pass the maximum taken by this many powers of two
// Workgroups asked for (two a compute unit; 4 images of 16384 keys, 16 heads: 82 us with three, 77 with
// two, 97 with one) and the fewest 32-key tiles a wave is left with.
constexpr long kGroups = 512;
constexpr int kLeastTiles = 2;

template <class S, int DH>
constexpr int wave_bytes()
{
    return 32 * Tile<S, DH>::kRowBytes + 32 * 8;
}

// Partial results: (maximum, sum, sum of what was multiplied, nothing; DH outputs) a column.
template <int DH>
constexpr int part_floats()
{
    return DH + 4;
}

// Four outputs of a column from its joined sums (by: of what was multiplied), rounded once, and its statistics.
template <class S>
__device__ __forceinline__ void store_column(uint8_t* row, float4 o, float top, float total, float by, int d, int dh,
                                             float* lse, S)
{
    const float inv = by > 0.0f ? 1.0f / by : (by == 0.0f ? 0.0f : by);  // no key: zeros
    if (d < dh) {
        if constexpr (S::kBytes == 2) {
            const f32x2 lo = {o.x * inv, o.y * inv}, hi = {o.z * inv, o.w * inv};
            uint2 w;
            w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2));
            w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2));
            *reinterpret_cast<uint2*>(row + d * 2) = w;
        } else {
            *reinterpret_cast<float4*>(row + d * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        }
    }
    if (lse && d == 0)
        *reinterpret_cast<float2*>(lse) =
            total == 0.0f ? make_float2(-__builtin_inff(), 0.0f) : make_float2(top, __builtin_log2f(total));
}

// Waves a SIMD the registers are held to: three (bfloat16, 64 channels: 64 images of up to 4096 keys, one
// query each, 165 us with two, 149 with three) where no key bias is carried along, which then spills
// (4 images of 16384 keys: 71 us with two, 93 with three).
template <class S, int DH, bool KB>
constexpr int waves_per_simd()
{
    return S::kBytes == 2 && DH == 64 && !KB ? 3 : 2;
}

template <class S, int DH, int BIAS, bool KB>
__global__ __launch_bounds__(kThreads, (waves_per_simd<S, DH, KB>())) void attention_few_kernel(AttentionCall a, HeadRows q, HeadRows k, HeadRows v,
                                                                   HeadRows out, float* __restrict__ lse,
                                                                   float* __restrict__ parts, int splits)
{
    typedef Tile<S, DH> T;
    typedef typename FragOf<S>::type Frag;
    constexpr int kChunksLane = 32 * T::kChunks / kWave;
    constexpr int kPad = DH + 4;
    extern __shared__ __align__(16) uint8_t lds[];
    const int split = blockIdx.x % splits, pair = blockIdx.x / splits;
    const int b = pair / a.Hk, hk = pair - b * a.Hk, group = a.H / a.Hk;
    const Rows rq = image_rows(a.q_off, b, a.Nq), rk = image_rows(a.k_off, b, a.Nk);
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, l32 = lane & 31, h = lane >> 5;
    const int hd = hk * group + l32 / a.Nq, qi = l32 % a.Nq;  // this lane's column
    const bool live = l32 < group * a.Nq && qi < rq.count;
    const int W = 2 * a.span + 1;
    const float c = a.scale * kLog2e;
    // The tiles of this workgroup, dealt to its waves in turn.
    const int tiles = (rk.count + 31) / 32;
    const int t0 = (int)((long)tiles * split / splits), t1 = (int)((long)tiles * (split + 1) / splits);

    uint8_t* vt = lds + wave * wave_bytes<S, DH>();
    int* codes = reinterpret_cast<int*>(vt + 32 * T::kRowBytes);
    float* kbs = reinterpret_cast<float*>(codes + 32);

    Frag qf[DH / 16], kf[DH / 16];
    u32x4 vn[kChunksLane];
    int pos = 0;
    float kbias = 0.0f, bn[16];
    auto load_positions = [&](int tile) {
        const int kk = 32 * tile + l32;
        pos = kk < rk.count ? (a.k_pos ? a.k_pos[rk.first + kk] : kk) : 0;
    };
    const bool biased = BIAS != kBiasNone && live;
    int qcode = 0;
    const uint8_t* bias = nullptr;
    // The bias entries of the tile whose positions are there: their codes go through LDS, as each lane
    // reads those of 16 keys for its column.
    auto load_bias = [&]() {
        if (h == 0) codes[l32] = bias_code<BIAS>(pos, a.grid_h, a.grid_w, W);
        __builtin_amdgcn_wave_barrier();
        if (biased) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const i32x4 kc = *reinterpret_cast<const i32x4*>(codes + 8 * g + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    bn[4 * g + e] = *reinterpret_cast<const float*>(bias + bias_entry<BIAS>(qcode, kc[e], a.span, W, 0));
            }
        }
        __builtin_amdgcn_wave_barrier();
    };
    auto load = [&](int tile) {
        const int kk = 32 * tile + l32;
        const bool in = kk < rk.count;
        if (KB) kbias = in ? a.k_bias[rk.first + kk] : -__builtin_inff();
        const long row = rk.first + (in ? kk : 0);
        load_frags<S, DH>(kf, k.p + (row * k.row + (long)hk * k.head) * S::kBytes, a.dh, in, h);
#pragma unroll
        for (int i = 0; i < kChunksLane; ++i) {
            const int e = lane + i * kWave, ch = e % T::kChunks, kv = 32 * tile + e / T::kChunks;
            const bool have = kv < rk.count;
            vn[i] = load_chunk<S>(v.p + ((rk.first + (have ? kv : 0)) * v.row + (long)hk * v.head) * S::kBytes, ch, a.dh,
                                  have);
        }
    };
    const int first = t0 + wave;
    if (BIAS != kBiasNone && first < t1) load_positions(first);
    const long qrow = rq.first + (live ? qi : 0);
    load_frags<S, DH>(qf, q.p + (qrow * q.row + (long)(live ? hd : 0) * q.head) * S::kBytes, a.dh, live, h);
    if (BIAS != kBiasNone) {
        qcode = query_code<BIAS>(live ? (a.q_pos ? a.q_pos[qrow] : qi) : 0, a.grid_h, a.grid_w, a.span, W, 0);
        bias = reinterpret_cast<const uint8_t*>(a.bias + (long)(live ? hd : 0) * W * W);
    }
    if (first < t1) {
        load(first);
        if (BIAS != kBiasNone) {
            load_bias();
            if (first + kWaves < t1) load_positions(first + kWaves);
        }
    }
    f32x16 acc[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.0f;
    float m = -__builtin_inff(), sum = 0.0f, used = 0.0f;  // (used: as in the kernel of many queries)

    for (int tile = first; tile < t1; tile += kWaves) {
#pragma unroll
        for (int i = 0; i < kChunksLane; ++i) {
            const int e = lane + i * kWave;
            if (KB && __shfl(kbias, e / T::kChunks) == -__builtin_inff()) {  // dropped: whatever it holds
                const u32x4 zero = {0, 0, 0, 0};
                vn[i] = zero;
            }
            store16(vt + T::at(e / T::kChunks, e % T::kChunks), vn[i]);
        }
        if (KB && h == 0) kbs[l32] = to_log2(kbias);
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
        for (int st = 0; st < DH / 16; ++st) {
            if (KB && kbias == -__builtin_inff()) kf[st] = Frag{};
            s = mma(kf[st], qf[st], s);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = BIAS != kBiasNone ? fmaf(s[r], c, biased ? to_log2(bn[r]) : 0.0f) : s[r] * c;
        // What the next tile needs goes out here, and the positions of the one after: loads return in
        // order, so that one wait a tile covers all of them.
        if (tile + kWaves < t1) {
            if (BIAS != kBiasNone) load_bias();
            if (BIAS != kBiasNone && tile + 2 * kWaves < t1) load_positions(tile + 2 * kWaves);
            load(tile + kWaves);
        }
        __builtin_amdgcn_wave_barrier();  // one wave's own LDS: in order

        float top = -__builtin_inff();
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            f32x4 kb = {0, 0, 0, 0};
            if (KB) kb = *reinterpret_cast<const f32x4*>(kbs + 8 * g + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = s[4 * g + e];
                if (KB) x = kb[e] == -__builtin_inff() ? kb[e] : x + kb[e];
                else if (32 * tile + 8 * g + 4 * h + e >= rk.count) x = -__builtin_inff();
                s[4 * g + e] = x;
                top = fmaxf(top, x);
            }
        }
        top = halves_max(top);
        if (__any(top > (m == -__builtin_inff() ? m : m + kSlack))) {
            const float up = fmaxf(m, top);
            const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - up);
            m = up;
            sum *= f;
            if (S::kBytes == 2) used *= f;
#pragma unroll
            for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[d][r] *= f;
        }
        const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(s[r] - base);
            sum += s[r];
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const Frag p = tile_frag(s, st, S{});
            used = frag_sum(p, used);
#pragma unroll
            for (int d = 0; d < DH / 32; ++d) acc[d] = mma(cols_frag<S, DH>(vt, 16 * st, 32 * d, lane), p, acc[d]);
        }
        __builtin_amdgcn_wave_barrier();
    }
    sum = halves_sum(sum);
    used = S::kBytes == 2 ? halves_sum(used) : sum;

    // The waves' results meet in LDS: (maximum, sums) and outputs of every column.
    __syncthreads();
    float* ms = reinterpret_cast<float*>(lds);
    float* outs = ms + kWaves * kCols * 4;
    if (h == 0) reinterpret_cast<float4*>(ms)[wave * kCols + l32] = make_float4(m, sum, used, 0.0f);
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4*>(outs + (wave * kCols + l32) * kPad + 32 * d + 8 * g + 4 * h) =
                make_float4(acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]);
    __syncthreads();
    const int per = DH / 4;  // threads a column, four outputs each
    for (int i = t; i < group * a.Nq * per; i += kThreads) {
        const int col = i / per, d = i % per * 4, q_i = col % a.Nq, head = hk * group + col / a.Nq;
        if (q_i >= rq.count) continue;
        float top = -__builtin_inff(), total = 0.0f, by = 0.0f;
        float4 o = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ms[4 * (w * kCols + col)]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float4 s = reinterpret_cast<const float4*>(ms)[w * kCols + col];
            const float f = s.x == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(s.x - top);
            const float4 x = *reinterpret_cast<const float4*>(outs + (w * kCols + col) * kPad + d);
            total += f * s.y;
            by += f * s.z;
            o = make_float4(fmaf(f, x.x, o.x), fmaf(f, x.y, o.y), fmaf(f, x.z, o.z), fmaf(f, x.w, o.w));
        }
        if (splits > 1) {
            float* part = parts + (((long)pair * splits + split) * group * a.Nq + col) * part_floats<DH>();
            if (d == 0) *reinterpret_cast<float4*>(part) = make_float4(top, total, by, 0.0f);
            *reinterpret_cast<float4*>(part + 4 + d) = o;
            continue;
        }
        store_column(out.p + ((rq.first + q_i) * out.row + (long)head * out.head) * S::kBytes, o, top, total, by, d, a.dh,
                     lse ? lse + 2 * ((rq.first + q_i) * a.H + head) : nullptr, S{});
    }
}

// Joins the splits of a column: a thread four outputs of one, splits in order.
template <class S, int DH>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(AttentionCall a, HeadRows out, float* __restrict__ lse,
                                                                  const float* __restrict__ parts, int splits)
{
    constexpr int kPer = DH / 4;
    const int group = a.H / a.Hk, cols = group * a.Nq;
    const long i = (long)blockIdx.x * kThreads + threadIdx.x;
    const long column = i / kPer;
    const int d = (int)(i % kPer) * 4;
    if (column >= (long)a.B * a.Hk * cols) return;
    const int pair = (int)(column / cols), col = (int)(column % cols), b = pair / a.Hk;
    const int q_i = col % a.Nq, head = (pair - b * a.Hk) * group + col / a.Nq;
    const Rows rq = lane_rows(a.q_off, b, a.Nq);
    if (q_i >= rq.count) return;
    const float* part = parts + ((long)pair * splits * cols + col) * part_floats<DH>();
    const long step = (long)cols * part_floats<DH>();
    float top = -__builtin_inff(), total = 0.0f, by = 0.0f;
    for (int s = 0; s < splits; ++s) top = fmaxf(top, part[s * step]);
    float4 o = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float* p = part + s * step;
        const float f = p[0] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(p[0] - top);
        const float4 x = *reinterpret_cast<const float4*>(p + 4 + d);
        total += f * p[1];
        by += f * p[2];
        o = make_float4(fmaf(f, x.x, o.x), fmaf(f, x.y, o.y), fmaf(f, x.z, o.z), fmaf(f, x.w, o.w));
    }
    store_column(out.p + ((rq.first + q_i) * out.row + (long)head * out.head) * S::kBytes, o, top, total, by, d, a.dh,
                 lse ? lse + 2 * ((rq.first + q_i) * a.H + head) : nullptr, S{});
}

template <class S, int DH, int BIAS, bool KB>
hipError_t launch(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v, const HeadRows& out,
                  float* lse, float* parts, hipStream_t st)
{
    const int splits = attention_few_splits(a);
    const size_t joined = kWaves * kCols * (4 + DH + 4) * 4;
    const size_t bytes = std::max((size_t)kWaves * wave_bytes<S, DH>(), joined);
    const long pairs = (long)a.B * a.Hk;
    if (pairs * splits * kThreads > UINT32_MAX) return hipErrorInvalidConfiguration;
    auto kernel = attention_few_kernel<S, DH, BIAS, KB>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(pairs * splits)), dim3(kThreads), bytes, st, a, q, k, v, out, lse, parts,
                       splits);
    e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    const long threads = pairs * (a.H / a.Hk) * a.Nq * (DH / 4);
    hipLaunchKernelGGL((attention_join_kernel<S, DH>), dim3((unsigned)((threads + kThreads - 1) / kThreads)),
                       dim3(kThreads), 0, st, a, out, lse, parts, splits);
    return hipGetLastError();
}

template <class S, int DH>
hipError_t pick(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v, const HeadRows& out,
                float* lse, float* parts, hipStream_t st)
{
    const int bias = bias_kind(a);
    if (a.k_bias) {
        if (bias == kBiasNone) return launch<S, DH, kBiasNone, true>(a, q, k, v, out, lse, parts, st);
        if (bias == kBiasGrid) return launch<S, DH, kBiasGrid, true>(a, q, k, v, out, lse, parts, st);
        return launch<S, DH, kBiasFar, true>(a, q, k, v, out, lse, parts, st);
    }
    if (bias == kBiasNone) return launch<S, DH, kBiasNone, false>(a, q, k, v, out, lse, parts, st);
    if (bias == kBiasGrid) return launch<S, DH, kBiasGrid, false>(a, q, k, v, out, lse, parts, st);
    return launch<S, DH, kBiasFar, false>(a, q, k, v, out, lse, parts, st);
}

}  // namespace

// The queries of the heads that share a key head fit a tile's columns. Tiles of queries instead (12 heads,
// one query an image, us there / here): 4 images of 16384 keys, 16 heads 477 / 71, 64 of up to 4096
// 330 / 149, 64 of up to 1024 43 / 41, 64 of 256 24 / 26, one of up to 1024 26 / 23; 20 queries an image:
// 64 of up to 4096 331 / 204, 64 of up to 1024 44 / 55. Heads of 128: 64 of up to 4096 511 / 399, of up to 1024
// 147 / 116, of up to 256 44 / 47; float32: 16 of up to 4096 224 / 101, 64 of up to 1024 188 / 105, of up to 256 62 / 45;
// float32 heads of 128: 1340 / 682, 1004 / 656, 204 / 217.
bool attention_is_few(const AttentionCall& a) { return (long)a.H / a.Hk * a.Nq <= kCols; }

int attention_few_splits(const AttentionCall& a)
{
    const long pairs = (long)a.B * a.Hk, tiles = (a.Nk + 31) / 32;
    const long most = std::max(1L, tiles / (kWaves * kLeastTiles));
    return (int)std::max(1L, std::min((kGroups + pairs - 1) / pairs, most));
}

size_t attention_few_bytes(const AttentionCall& a)
{
    const int splits = attention_few_splits(a);
    if (splits == 1) return 0;
    return (size_t)a.B * a.H * a.Nq * splits * (a.dh <= 64 ? part_floats<64>() : part_floats<128>()) * 4;
}

hipError_t launch_attention_few(const AttentionCall& a, const HeadRows& q, const HeadRows& k, const HeadRows& v,
                                const HeadRows& out, float* lse, void* ws, hipStream_t st)
{
    float* parts = static_cast<float*>(ws);
    if (a.dt == kBf16)
        return a.dh <= 64 ? pick<Bf16, 64>(a, q, k, v, out, lse, parts, st) : pick<Bf16, 128>(a, q, k, v, out, lse, parts, st);
    return a.dh <= 64 ? pick<F32, 64>(a, q, k, v, out, lse, parts, st) : pick<F32, 128>(a, q, k, v, out, lse, parts, st);
}

}  // namespace mpm

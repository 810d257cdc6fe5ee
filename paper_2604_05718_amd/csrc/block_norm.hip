// The norms around a transformer block with the block's gate, residual scale and residual sum:
//   u = post(f) or f,   y = x + scale * gate * u,   h = pre(y),
// post and pre each a layer norm ((t - mean) rstd w + b) or a root-mean-square norm (t rstd w),
// and the gradients of all of it. Bound by memory: forward reads x and f and writes y and h,
// backward reads dy, dh, y and f and writes dx and df; everything between stays in registers. Rows of
// the next turn load while one is computed. Layer norms on both sides, bfloat16: 64 images of about 717
// rows of 768 (282 MB) 60 us forward, 4.7 TB/s; 16 of about 2870 rows of 1024 (376 and 564 MB) 68 us forward,
// 5.5 TB/s, and 137 us backward, 4.1 TB/s, with 6 us to join the column sums: the backward's two norms
// are four sums of a row one after another, which two waves a SIMD do not hide in full (registers held
// to three or four spill: a step 219 -> 552 and 742 us). Rows of 1024 threads (more than 4096 bfloat16 values or
// 2048 float32) leave 128 registers a lane: the backward kernel keeps up to 1132 bytes a lane in scratch memory,
// the forward one up to 312.
//
// The backward pass norms y as it was stored, rounded to its type: in bfloat16 an error of 2^-9 of a value that
// the weight's gradient shows (0.0023 of its norm against 0.0017), and that grows with a row's mean over its deviation.
#include <algorithm>
#include <type_traits>

#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {
namespace {

constexpr int kMinThreads = 256;
// Workgroups of the column sums: enough to fill the chip, few enough that their partial sums
// (a few rows of D floats each) are small beside the rows.
constexpr int kSumGroups = 512;
// Workgroups of the forward kernel: a few rows for each row group, so that loads run ahead.
constexpr int kForwardGroups = 2048;
// Half as many of both / these / twice as many: 64 images of about 717 rows of 768, forward, 71 / 70 / 72 us; a
// step of 16 of about 2870 rows of 1024 239 / 238 / 262; float32, 7 of about 670 rows of 836, 50 / 52 / 58.
constexpr int kSums = 5;  // dw, db, dscale, dpost_w, dpost_b (a gate's sums are by image)

template <class S>
__device__ __forceinline__ u32x4 pack(const float* v)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (S::kBytes == 2) {
            const f32x2 p = {v[2 * e], v[2 * e + 1]};
            r[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        } else {
            r[e] = __float_as_uint(v[e]);
        }
    }
    return r;
}

// Threads of a workgroup for LANES lanes a row.
template <int LANES>
constexpr int threads()
{
    return LANES > kMinThreads ? LANES : kMinThreads;
}

// A value plus its counterpart's by a fixed lane pattern inside 16 lanes.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}

// The sum of a value over 32 or 64 lanes, in every lane: exchanges inside 16 lanes (neighbour, pair,
// half and whole mirror), then between the 16s and the 32s. No LDS: two sums of a row by LDS
// exchanges took a third of a row's time.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    v = dpp_add<0xb1>(v);   // lane ^ 1
    v = dpp_add<0x4e>(v);   // lane ^ 2
    v = dpp_add<0x141>(v);  // 7 - lane of 8
    v = dpp_add<0x140>(v);  // 15 - lane of 16
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    if constexpr (LANES >= kWave) {
        const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(q[0]) + __uint_as_float(q[1]);
    }
    return v;
}

// The sums of two values over the lanes of a row, in a fixed order. Rows of several waves meet in LDS:
// every row group of the workgroup has to call.
template <int LANES>
__device__ __forceinline__ void row_sums(float& a, float& b, float* lds)
{
    a = lanes_sum<LANES>(a);
    b = lanes_sum<LANES>(b);
    if constexpr (LANES > kWave) {
        constexpr int kWaves = LANES / kWave;
        const int wave = threadIdx.x / kWave, first = wave / kWaves * kWaves;
        __syncthreads();  // the sums before have been read
        if (threadIdx.x % kWave == 0) {
            lds[2 * wave] = a;
            lds[2 * wave + 1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            a += lds[2 * (first + w)];
            b += lds[2 * (first + w) + 1];
        }
    }
}

// A row's part in one lane as it is stored: VPL vectors of 16 bytes, vector lane + u LANES of the row.
template <class S, int LANES, int VPL>
struct RawPart {
    static constexpr int kPer = 16 / S::kBytes;
    static constexpr int kVals = VPL * kPer;
    u32x4 v[VPL];

    // A row's vectors. Lanes past the row's end read its last vector again (`in` tells them apart), so
    // that loads are never behind a branch.
    __device__ __forceinline__ void load(const void* base, long row, int D, int lane)
    {
        const uint8_t* p = static_cast<const uint8_t*>(base) + row * D * S::kBytes;
        const int last = D / kPer - 1;
#pragma unroll
        for (int u = 0; u < VPL; ++u) v[u] = load16(p + min(lane + u * LANES, last) * 16);
    }
    // A row of parameters: zeros past the row's end; `missing` where there is none.
    __device__ __forceinline__ void param(const void* base, long row, int D, int lane, float missing)
    {
        const uint32_t word = S::kBytes == 2 ? f32_to_bf16_rne(missing) * 0x10001u : __float_as_uint(missing);
        const uint8_t* p = static_cast<const uint8_t*>(base) + row * D * S::kBytes;
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
            const int c = lane + u * LANES;
            const uint32_t fill = c * kPer < D ? word : 0;
            const u32x4 none = {fill, fill, fill, fill};
            v[u] = none;
            if (base && c * kPer < D) v[u] = load16(p + c * 16);
        }
    }
    __device__ __forceinline__ void clear()
    {
        const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < VPL; ++u) v[u] = zero;
    }
    __device__ __forceinline__ float get(int e) const
    {
        const u32x4 w = v[e / kPer];
        const int k = e % kPer;
        if constexpr (S::kBytes == 2) return k % 2 ? bf16_hi(w[k / 2]) : bf16_lo(w[k / 2]);
        return __uint_as_float(w[k]);
    }
    // Whether value e of this lane lies inside the row.
    __device__ static __forceinline__ bool in(int e, int lane, int D) { return (lane + e / kPer * LANES) * kPer < D; }
    __device__ static __forceinline__ void store(const float (&x)[kVals], void* base, long row, int D, int lane)
    {
        uint8_t* p = static_cast<uint8_t*>(base) + row * D * S::kBytes;
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
            const int c = lane + u * LANES;
            if (c * kPer < D) store16(p + c * 16, pack<S>(x + u * kPer));
        }
    }
};

struct Item {
    long first, end;  // rows
    int image;
};
// Work item i of images x chunks: chunk i % chunks of image i / chunks' rows.
__device__ __forceinline__ Item item_rows(const NormCall& a, long i)
{
    const int b = (int)(i / a.chunks), c = (int)(i % a.chunks);
    const long lo = a.off ? a.off[b] : (long)b * a.N;
    const long hi = a.off ? a.off[b + 1] : lo + a.N;
    const long first = min(max(lo, 0L), (long)a.R), n = min(max(hi, first), (long)a.R) - first;
    return Item{first + n * c / a.chunks, first + n * (c + 1) / a.chunks, b};
}

// Mean and reciprocal deviation of a row's values (rms: mean 0).
template <class S, int LANES, int VPL>
__device__ __forceinline__ void row_stats(const float (&x)[RawPart<S, LANES, VPL>::kVals], int D, int lane, bool layer,
                                          float eps, float* lds, float& mean, float& rstd)
{
    typedef RawPart<S, LANES, VPL> Raw;
    mean = 0.0f;
    float none = 0.0f;
    if (layer) {
#pragma unroll
        for (int e = 0; e < Raw::kVals; ++e) mean += Raw::in(e, lane, D) ? x[e] : 0.0f;
        row_sums<LANES>(mean, none, lds);
        mean /= (float)D;
    }
    float sq = 0.0f;
#pragma unroll
    for (int e = 0; e < Raw::kVals; ++e) {
        const float d = Raw::in(e, lane, D) ? x[e] - mean : 0.0f;
        sq = fmaf(d, d, sq);
    }
    none = 0.0f;
    row_sums<LANES>(sq, none, lds);
    rstd = 1.0f / sqrtf(sq / (float)D + eps);
}

// What a kernel is compiled for: a norm after the block, a norm before the next one.
// Parameters that are not given are ones (scale, gate) or zeros (shifts).
//
// Forward: a row group of LANES lanes takes every kRows-th row of the workgroup's, the next row's x and
// f on their way while one is computed; the parameters stay in registers. y may be x itself: a row is loaded
// before it is stored, and what is loaded of it again past the workgroup's end is not used.
template <class S, int LANES, int VPL, bool POST, bool PRE>
__global__ __launch_bounds__(threads<LANES>()) void norm_kernel(NormCall a, const void* x,
                                                               const void* __restrict__ f, void* y,
                                                               void* __restrict__ hout, float* __restrict__ stats)
{
    typedef RawPart<S, LANES, VPL> Raw;
    __shared__ float lds[2 * threads<LANES>() / kWave];
    constexpr int kRows = threads<LANES>() / LANES, kVals = Raw::kVals;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, D = a.D;
    const Item it = item_rows(a, blockIdx.x);
    if (it.first >= it.end) return;
    Raw fn, xn, pw, pb, sc, ga, w, b;
    fn.load(f, min(it.first + sub, it.end - 1), D, lane);
    xn.load(x, min(it.first + sub, it.end - 1), D, lane);
    if (POST) {
        pw.param(a.post_w, 0, D, lane, 0.0f);
        pb.param(a.post_b, 0, D, lane, 0.0f);
    }
    sc.param(a.scale, 0, D, lane, 1.0f);
    ga.param(a.gate_rows ? nullptr : a.gate, it.image, D, lane, 1.0f);
    if (PRE) {
        w.param(a.w, 0, D, lane, 0.0f);
        b.param(a.b, 0, D, lane, 0.0f);
    }
    for (long base = it.first; base < it.end; base += kRows) {
        const long row = min(base + sub, it.end - 1);
        const bool live = base + sub < it.end;
        float u[kVals], r[kVals];
#pragma unroll
        for (int e = 0; e < kVals; ++e) {
            u[e] = fn.get(e);
            r[e] = xn.get(e);
        }
        if (a.gate_rows) ga.load(a.gate, row, D, lane);
        const long next = min(base + sub + kRows, it.end - 1);
        fn.load(f, next, D, lane);
        xn.load(x, next, D, lane);
        float pmean = 0.0f, prstd = 1.0f;
        if (POST) {
            row_stats<S, LANES, VPL>(u, D, lane, a.layer, a.eps, lds, pmean, prstd);
#pragma unroll
            for (int e = 0; e < kVals; ++e) u[e] = fmaf((u[e] - pmean) * prstd, pw.get(e), pb.get(e));
        }
#pragma unroll
        for (int e = 0; e < kVals; ++e) r[e] = fmaf(u[e] * sc.get(e), ga.get(e), r[e]);
        if (live) Raw::store(r, y, row, D, lane);
        float mean = 0.0f, rstd = 1.0f;
        if (PRE) {
            // Of the sum before its rounding to y's type, which only the stored y has.
            row_stats<S, LANES, VPL>(r, D, lane, a.layer, a.eps, lds, mean, rstd);
#pragma unroll
            for (int e = 0; e < kVals; ++e) r[e] = fmaf((r[e] - mean) * rstd, w.get(e), b.get(e));
            if (live) Raw::store(r, hout, row, D, lane);
        }
        if (stats && live && lane == 0) reinterpret_cast<float4*>(stats)[row] = make_float4(pmean, prstd, mean, rstd);
    }
}

// Adds a workgroup's column sums (its row groups in order) and stores them as row `slot` of out.
template <class S, int LANES, int VPL>
__device__ __forceinline__ void store_sums(const float* v, float* out, long slot, int D, int lane, int sub, float* lds)
{
    typedef RawPart<S, LANES, VPL> Part;
    constexpr int kRows = threads<LANES>() / LANES;
    if constexpr (kRows > 1) __syncthreads();
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
        const int c = lane + u * LANES;
#pragma unroll
        for (int e = 0; e < Part::kPer; ++e) {
            float s = v[u * Part::kPer + e];
            if constexpr (kRows > 1) {
                lds[sub * LANES + lane] = s;
                __syncthreads();
                if (sub == 0) {
#pragma unroll
                    for (int k = 1; k < kRows; ++k) s += lds[k * LANES + lane];
                }
                __syncthreads();
            }
            if (sub == 0 && c * Part::kPer < D) out[slot * D + c * Part::kPer + e] = s;
        }
    }
}

// dx and df of every row, and the workgroup's column sums: sums[k][group][D] (kSums of them) and, for
// a gate by image, gate_sums[item][D]. Rows and parameters as in the forward kernel.
//
// With u = post_w t + post_b and g the gradient of y, every parameter beside the block is a combination of two
// sums over rows, A = sum of gate g t and B = sum of gate g: dpost_w = scale A, dpost_b = scale B, dscale =
// post_w A + post_b B, and an image's dgate = scale (post_w A' + post_b B') from its own, ungated. A row
// costs two sums a value instead of four and their factors (a step of 16 images of about 2870 rows of
// 1024, bfloat16: 234 -> 219 us).
template <class S, int LANES, int VPL, bool POST, bool PRE, bool GATE_ROWS>
__global__ __launch_bounds__(threads<LANES>()) void norm_backward_kernel(
    NormCall a, const void* __restrict__ dy, const void* __restrict__ dh, const void* __restrict__ y,
    const void* __restrict__ f, const float* __restrict__ stats, void* __restrict__ dx, void* __restrict__ df,
    void* __restrict__ dgate, float* __restrict__ sums, float* __restrict__ gate_sums, long items)
{
    typedef RawPart<S, LANES, VPL> Raw;
    constexpr int kRows = threads<LANES>() / LANES, kVals = Raw::kVals;
    __shared__ float lds[threads<LANES>()];
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, D = a.D;
    const float inv = 1.0f / (float)D, centred = a.layer ? inv : 0.0f;
    float sw[kVals], sb[kVals], sa[kVals], sg[kVals];  // sa, sg: A and B
#pragma unroll
    for (int e = 0; e < kVals; ++e) sw[e] = sb[e] = sa[e] = sg[e] = 0.0f;
    Raw w, pw, pb, sc, ga;
    if (PRE) w.param(a.w, 0, D, lane, 0.0f);
    if (POST) {
        pw.param(a.post_w, 0, D, lane, 0.0f);
        pb.param(a.post_b, 0, D, lane, 0.0f);
    }
    sc.param(a.scale, 0, D, lane, 1.0f);
    for (long i = blockIdx.x; i < items; i += gridDim.x) {
        const Item it = item_rows(a, i);
        float ia[kVals], ig[kVals], factor[kVals];  // the item's sums; of g t in the gradient of t
        ga.param(GATE_ROWS ? nullptr : a.gate, it.image, D, lane, 1.0f);
#pragma unroll
        for (int e = 0; e < kVals; ++e) {
            ia[e] = ig[e] = 0.0f;
            factor[e] = sc.get(e) * ga.get(e) * (POST ? pw.get(e) : 1.0f);  // POST: zero past the row's end
        }
        Raw yn, hn, gn, fn;
        float4 stn;
        auto load = [&](long at) {
            const long row = min(at, it.end - 1);
            if (dy) gn.load(dy, row, D, lane);
            if (PRE) {
                yn.load(y, row, D, lane);
                hn.load(dh, row, D, lane);
            }
            fn.load(f, row, D, lane);
            stn = reinterpret_cast<const float4*>(stats)[row];
        };
        if (!dy) gn.clear();
        if (it.first < it.end) load(it.first + sub);
        // Every row group takes the same number of turns: the sums of a row of several waves meet
        // at barriers.
        for (long base = it.first; base < it.end; base += kRows) {
            const bool live = base + sub < it.end;
            const long row = live ? base + sub : it.end - 1;
            if (!live) {  // a row past the end adds nothing to the sums
                gn.clear();
                hn.clear();
            }
            const float4 st = stn;
            if (GATE_ROWS) ga.load(a.gate, row, D, lane);
            float g[kVals], t[kVals], n[kVals];
            if (PRE) {
#pragma unroll
                for (int e = 0; e < kVals; ++e) {
                    n[e] = (yn.get(e) - st.z) * st.w;
                    t[e] = hn.get(e);
                }
            }
            const Raw fr = fn;
#pragma unroll
            for (int e = 0; e < kVals; ++e) g[e] = gn.get(e);
            load(base + sub + kRows);
            if (PRE) {
                float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
                for (int e = 0; e < kVals; ++e) {
                    sb[e] += t[e];
                    sw[e] = fmaf(t[e], n[e], sw[e]);
                    t[e] *= w.get(e);  // zero past the row's end
                    m1 += t[e];
                    m2 = fmaf(t[e], n[e], m2);
                }
                row_sums<LANES>(m1, m2, lds);
                m1 *= -st.w * centred;
                m2 *= -st.w * inv;
#pragma unroll
                for (int e = 0; e < kVals; ++e) g[e] += fmaf(st.w, t[e], fmaf(n[e], m2, m1));
            }
            if (live) Raw::store(g, dx, row, D, lane);
            // t: the unit rows of f (or f)
#pragma unroll
            for (int e = 0; e < kVals; ++e) t[e] = POST ? (fr.get(e) - st.x) * st.y : fr.get(e);
            if (!live) {
#pragma unroll
                for (int e = 0; e < kVals; ++e) g[e] = 0.0f;
            }
            float n1 = 0.0f, n2 = 0.0f;
#pragma unroll
            for (int e = 0; e < kVals; ++e) {
                if (GATE_ROWS) {
                    n[e] = g[e] * (sc.get(e) * (POST ? fmaf(t[e], pw.get(e), pb.get(e)) : t[e]));
                    g[e] *= ga.get(e);
                }
                ia[e] = fmaf(g[e], t[e], ia[e]);
                if (POST) ig[e] += g[e];
                g[e] *= factor[e];
                if (POST) {
                    n1 += g[e];
                    n2 = fmaf(g[e], t[e], n2);
                }
            }
            if (GATE_ROWS && live) Raw::store(n, dgate, row, D, lane);
            if (POST) {
                row_sums<LANES>(n1, n2, lds);
                n1 *= -st.y * centred;
                n2 *= -st.y * inv;
#pragma unroll
                for (int e = 0; e < kVals; ++e) g[e] = fmaf(st.y, g[e], fmaf(t[e], n2, n1));
            }
            if (live) Raw::store(g, df, row, D, lane);
        }
#pragma unroll
        for (int e = 0; e < kVals; ++e) {
            const float gate = GATE_ROWS ? 1.0f : ga.get(e);
            sa[e] = fmaf(gate, ia[e], sa[e]);
            if (POST) sg[e] = fmaf(gate, ig[e], sg[e]);
            ia[e] = sc.get(e) * (POST ? fmaf(pw.get(e), ia[e], pb.get(e) * ig[e]) : ia[e]);
        }
        if (gate_sums) store_sums<S, LANES, VPL>(ia, gate_sums, i, D, lane, sub, lds);
    }
    const long G = gridDim.x, at = blockIdx.x;
    if (PRE) {
        store_sums<S, LANES, VPL>(sw, sums, at, D, lane, sub, lds);
        if (a.b) store_sums<S, LANES, VPL>(sb, sums, G + at, D, lane, sub, lds);
    }
#pragma unroll
    for (int e = 0; e < kVals; ++e) {
        sw[e] = POST ? fmaf(pw.get(e), sa[e], pb.get(e) * sg[e]) : sa[e];
        sa[e] *= sc.get(e);
        sg[e] *= sc.get(e);
    }
    if (a.scale) store_sums<S, LANES, VPL>(sw, sums, 2 * G + at, D, lane, sub, lds);
    if (POST) {
        store_sums<S, LANES, VPL>(sa, sums, 3 * G + at, D, lane, sub, lds);
        if (a.post_b) store_sums<S, LANES, VPL>(sg, sums, 4 * G + at, D, lane, sub, lds);
    }
}

struct SumOut {
    void* p[kSums];
};

// The column sums of all workgroups: 16 threads a column take every 16th part, joined in order. Rows
// 0 ... kSums - 1 of the grid (in y and z: there may be more than a grid has in y): the parameters' (`groups`
// parts each), further rows: the gates of the images (`chunks` parts each). Columns along x, which is 1 us
// faster than rows along x (16 images, 1024 columns: 5.6 and 6.8 us).
constexpr int kGridRows = 32768;
__global__ __launch_bounds__(1024) void join_sums_kernel(const float* __restrict__ sums, int groups,
                                                         const float* __restrict__ gate_sums, int chunks, int rows, int D,
                                                         int dt, SumOut out, void* __restrict__ gate)
{
    constexpr int kCols = 64, kWays = 16;
    __shared__ float lds[kWays][kCols];
    const int col = blockIdx.x * kCols + threadIdx.x % kCols, way = threadIdx.x / kCols;
    const int row = blockIdx.z * kGridRows + blockIdx.y;
    if (row >= rows) return;
    const bool param = row < kSums;
    const long k = param ? row : row - kSums;
    void* dst = param ? out.p[k] : gate;
    if (dst == nullptr) return;
    const int parts = param ? groups : chunks;
    const float* from = (param ? sums : gate_sums) + k * parts * D + min(col, D - 1);
    float s = 0.0f;
#pragma unroll 8
    for (int g = way; g < parts; g += kWays) s += from[(long)g * D];
    lds[way][threadIdx.x % kCols] = s;
    __syncthreads();
    if (way != 0 || col >= D) return;
#pragma unroll
    for (int w = 1; w < kWays; ++w) s += lds[w][threadIdx.x];
    const long at = param ? col : k * D + col;
    if (dt == kBf16) reinterpret_cast<uint16_t*>(dst)[at] = (uint16_t)f32_to_bf16_rne(s);
    else reinterpret_cast<float*>(dst)[at] = s;
}

// Chunks an image for about `groups` workgroups, each of at least one row a row group.
int chunk_count(const NormCall& a, int groups, int rows)
{
    const long per = std::max(1L, ((long)a.R + a.B - 1) / a.B);
    return (int)std::max(1L, std::min(((long)groups + a.B - 1) / a.B, (per + rows - 1) / rows));
}

// Lanes a row: two vectors of 16 bytes a lane (four in the widest float32 rows), for registers that
// leave two waves a SIMD in the backward kernel.
template <class S, class F>
hipError_t with_lanes(int D, F&& go)
{
    const int vpr = D * S::kBytes / 16;
    constexpr std::integral_constant<int, 2> two{};
    if (vpr <= 64) return go(std::integral_constant<int, 32>{}, two);
    if (vpr <= 128) return go(std::integral_constant<int, 64>{}, two);
    if (vpr <= 256) return go(std::integral_constant<int, 128>{}, two);
    if (vpr <= 512) return go(std::integral_constant<int, 256>{}, two);
    if (vpr <= 2048) return go(std::integral_constant<int, 1024>{}, two);
    return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, S::kBytes>{});
}

// ... and the norms that are given.
template <class F>
hipError_t with_norms(const NormCall& a, F&& go)
{
    if (a.post_w) return a.w ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    return a.w ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
}

template <class S>
hipError_t forward(NormCall a, const void* x, const void* f, void* y, void* h, float* stats, hipStream_t st)
{
    return with_lanes<S>(a.D, [&](auto lanes, auto vpl) {
        return with_norms(a, [&](auto post, auto pre) {
            constexpr int L = decltype(lanes)::value, V = decltype(vpl)::value;
            constexpr bool POST = decltype(post)::value, PRE = decltype(pre)::value;
            a.chunks = chunk_count(a, kForwardGroups, threads<L>() / L);
            hipLaunchKernelGGL((norm_kernel<S, L, V, POST, PRE>), dim3((unsigned)((long)a.B * a.chunks)),
                               dim3(threads<L>()), 0, st, a, x, f, y, h, stats);
            return hipGetLastError();
        });
    });
}

int backward_chunks(const NormCall& a) { return chunk_count(a, kSumGroups, 4); }
long backward_groups(const NormCall& a) { return std::min((long)a.B * backward_chunks(a), (long)kSumGroups); }

template <class S>
hipError_t backward(NormCall a, const void* dy, const void* dh, const void* y, const void* f, const float* stats,
                    const NormGrads& g, float* sums, float* gate_sums, hipStream_t st)
{
    a.chunks = backward_chunks(a);
    const long items = (long)a.B * a.chunks, groups = backward_groups(a);
    const bool by_image = g.dgate && !a.gate_rows;
    hipError_t e = with_lanes<S>(a.D, [&](auto lanes, auto vpl) {
        return with_norms(a, [&](auto post, auto pre) {
            constexpr int L = decltype(lanes)::value, V = decltype(vpl)::value;
            constexpr bool POST = decltype(post)::value, PRE = decltype(pre)::value;
            auto kernel = a.gate_rows ? norm_backward_kernel<S, L, V, POST, PRE, true>
                                      : norm_backward_kernel<S, L, V, POST, PRE, false>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads<L>()), 0, st, a, dy, dh, y, f, stats, g.dx,
                               g.df, g.dgate, sums, by_image ? gate_sums : nullptr, items);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess) return e;
    const SumOut out{{g.dw, g.db, g.dscale, g.dpost_w, g.dpost_b}};
    if (!by_image && !g.dw && !g.dscale && !g.dpost_w) return e;
    const int rows = kSums + (by_image ? a.B : 0);
    hipLaunchKernelGGL(join_sums_kernel,
                       dim3((unsigned)((a.D + 63) / 64), (unsigned)std::min(rows, kGridRows),
                            (unsigned)((rows + kGridRows - 1) / kGridRows)),
                       dim3(1024), 0, st, sums, (int)groups, gate_sums, a.chunks, rows, a.D, a.dt, out,
                       by_image ? g.dgate : nullptr);
    return hipGetLastError();
}

size_t aligned256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

hipError_t launch_norm(const NormCall& a, const void* x, const void* f, void* y, void* h, float* stats, hipStream_t st)
{
    return a.dt == kBf16 ? forward<Bf16>(a, x, f, y, h, stats, st) : forward<F32>(a, x, f, y, h, stats, st);
}

size_t norm_backward_bytes(const NormCall& a)
{
    return aligned256((size_t)kSums * backward_groups(a) * a.D * 4) +
           aligned256((size_t)a.B * backward_chunks(a) * a.D * 4);
}

hipError_t launch_norm_backward(const NormCall& a, const void* dy, const void* dh, const void* y, const void* f,
                                const float* stats, const NormGrads& g, void* ws, hipStream_t st)
{
    float* sums = static_cast<float*>(ws);
    float* gate_sums = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                                aligned256((size_t)kSums * backward_groups(a) * a.D * 4));
    return a.dt == kBf16 ? backward<Bf16>(a, dy, dh, y, f, stats, g, sums, gate_sums, st)
                         : backward<F32>(a, dy, dh, y, f, stats, g, sums, gate_sums, st);
}

}  // namespace mpm

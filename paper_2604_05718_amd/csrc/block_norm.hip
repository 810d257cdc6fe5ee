// The norms around a transformer block with the block's gate, residual scale and residual sum:
//   u = post(f) or f,   y = x + scale * gate * u,   h = pre(y),
// post and pre each a layer norm ((t - mean) rstd w + b) or a root-mean-square norm (t rstd w),
// and the gradients of all of it. Bound by memory: forward reads x and f and writes y and h,
// backward reads dy, dh, y and f and writes dx and df; everything between stays in registers.
#include <algorithm>

#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {
namespace {

constexpr int kMinThreads = 256;
// Workgroups of the column sums: enough to fill the chip, few enough that their partial sums
// (a few rows of D floats each) are small beside the rows.
constexpr int kSumGroups = 512;
constexpr int kSums = 5;  // dw, db, dscale, dpost_w, dpost_b (a gate's sums are by image)

template <class S>
__device__ __forceinline__ void unpack(u32x4 v, float* out)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (S::kBytes == 2) {
            out[2 * e] = bf16_lo(v[e]);
            out[2 * e + 1] = bf16_hi(v[e]);
        } else {
            out[e] = __uint_as_float(v[e]);
        }
    }
}

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

// The sums of two values over the lanes of a row (in a fixed order).
template <int LANES>
__device__ __forceinline__ void row_sums(float& a, float& b, float* lds)
{
#pragma unroll
    for (int o = (LANES < kWave ? LANES : kWave) / 2; o > 0; o >>= 1) {
        a += __shfl_xor(a, o);
        b += __shfl_xor(b, o);
    }
    if constexpr (LANES > kWave) {
        constexpr int kWaves = LANES / kWave;
        const int wave = threadIdx.x / kWave;
        __syncthreads();  // the sums before have been read
        if (threadIdx.x % kWave == 0) {
            lds[2 * wave] = a;
            lds[2 * wave + 1] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            a += lds[2 * w];
            b += lds[2 * w + 1];
        }
    }
}

// A row's values in one lane: VPL vectors of 16 bytes, vector lane + u LANES of the row.
template <class S, int LANES, int VPL>
struct RowPart {
    static constexpr int kPer = 16 / S::kBytes;
    static constexpr int kVals = VPL * kPer;
    float v[kVals];

    __device__ __forceinline__ void load(const void* base, long row, int D, int lane)
    {
        const uint8_t* p = static_cast<const uint8_t*>(base) + row * D * S::kBytes;
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
            const int c = lane + u * LANES;
            u32x4 w = {0, 0, 0, 0};
            if (c * kPer < D) w = load16(p + c * 16);
            unpack<S>(w, v + u * kPer);
        }
    }
    __device__ __forceinline__ void fill(float x)
    {
#pragma unroll
        for (int e = 0; e < kVals; ++e) v[e] = x;
    }
    __device__ __forceinline__ void load_or(const void* base, long row, int D, int lane, float x)
    {
        if (base) load(base, row, D, lane);
        else fill(x);
    }
    __device__ __forceinline__ void store(void* base, long row, int D, int lane) const
    {
        uint8_t* p = static_cast<uint8_t*>(base) + row * D * S::kBytes;
#pragma unroll
        for (int u = 0; u < VPL; ++u) {
            const int c = lane + u * LANES;
            if (c * kPer < D) store16(p + c * 16, pack<S>(v + u * kPer));
        }
    }
    // Whether value e of this lane lies inside the row.
    __device__ static __forceinline__ bool in(int e, int lane, int D) { return (lane + e / kPer * LANES) * kPer < D; }
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
__device__ __forceinline__ void row_stats(const RowPart<S, LANES, VPL>& x, int D, int lane, bool layer, float eps,
                                          float* lds, float& mean, float& rstd)
{
    typedef RowPart<S, LANES, VPL> Part;
    mean = 0.0f;
    float none = 0.0f;
    if (layer) {
#pragma unroll
        for (int e = 0; e < Part::kVals; ++e) mean += x.v[e];  // zeros past the row's end
        row_sums<LANES>(mean, none, lds);
        mean /= (float)D;
    }
    float sq = 0.0f;
#pragma unroll
    for (int e = 0; e < Part::kVals; ++e) {
        const float d = Part::in(e, lane, D) ? x.v[e] - mean : 0.0f;
        sq = fmaf(d, d, sq);
    }
    none = 0.0f;
    row_sums<LANES>(sq, none, lds);
    rstd = 1.0f / sqrtf(sq / (float)D + eps);
}

template <class S, int LANES, int VPL>
__global__ __launch_bounds__(threads<LANES>()) void norm_kernel(NormCall a, const void* __restrict__ x,
                                                               const void* __restrict__ f, void* __restrict__ y,
                                                               void* __restrict__ hout, float* __restrict__ stats)
{
    typedef RowPart<S, LANES, VPL> Part;
    __shared__ float lds[2 * threads<LANES>() / kWave];
    constexpr int kRows = threads<LANES>() / LANES;
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, D = a.D;
    const Item it = item_rows(a, blockIdx.x);
    for (long row = it.first + sub; row < it.end; row += kRows) {
        Part u, r;
        float pmean = 0.0f, prstd = 1.0f;
        u.load(f, row, D, lane);
        r.load(x, row, D, lane);
        if (a.post_w) {
            row_stats(u, D, lane, a.layer, a.eps, lds, pmean, prstd);
            Part w, b;
            w.load(a.post_w, 0, D, lane);
            b.load_or(a.post_b, 0, D, lane, 0.0f);
#pragma unroll
            for (int e = 0; e < Part::kVals; ++e) u.v[e] = fmaf((u.v[e] - pmean) * prstd, w.v[e], b.v[e]);
        }
        if (a.scale) {
            Part w;
            w.load(a.scale, 0, D, lane);
#pragma unroll
            for (int e = 0; e < Part::kVals; ++e) u.v[e] *= w.v[e];
        }
        if (a.gate) {
            Part w;
            w.load(a.gate, a.gate_rows ? row : it.image, D, lane);
#pragma unroll
            for (int e = 0; e < Part::kVals; ++e) u.v[e] *= w.v[e];
        }
#pragma unroll
        for (int e = 0; e < Part::kVals; ++e) r.v[e] += u.v[e];
        r.store(y, row, D, lane);
        float mean = 0.0f, rstd = 1.0f;
        if (a.w) {
            // Of the sum before its rounding to y's type, which only the stored y has.
            row_stats(r, D, lane, a.layer, a.eps, lds, mean, rstd);
            Part w, b;
            w.load(a.w, 0, D, lane);
            b.load_or(a.b, 0, D, lane, 0.0f);
#pragma unroll
            for (int e = 0; e < Part::kVals; ++e) r.v[e] = fmaf((r.v[e] - mean) * rstd, w.v[e], b.v[e]);
            r.store(hout, row, D, lane);
        }
        if (stats && lane == 0) reinterpret_cast<float4*>(stats)[row] = make_float4(pmean, prstd, mean, rstd);
    }
}

// Adds a workgroup's column sums (its row groups in order) and stores them as row `slot` of out.
template <class S, int LANES, int VPL>
__device__ __forceinline__ void store_sums(const float* v, float* out, long slot, int D, int lane, int sub, float* lds)
{
    typedef RowPart<S, LANES, VPL> Part;
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
// a gate by image, gate_sums[item][D].
template <class S, int LANES, int VPL>
__global__ __launch_bounds__(threads<LANES>()) void norm_backward_kernel(
    NormCall a, const void* __restrict__ dy, const void* __restrict__ dh, const void* __restrict__ y,
    const void* __restrict__ f, const float* __restrict__ stats, void* __restrict__ dx, void* __restrict__ df,
    void* __restrict__ dgate, float* __restrict__ sums, float* __restrict__ gate_sums, long items)
{
    typedef RowPart<S, LANES, VPL> Part;
    constexpr int kRows = threads<LANES>() / LANES;
    __shared__ float lds[threads<LANES>()];
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, D = a.D;
    const float inv = 1.0f / (float)D;
    Part sw, sb, ss, spw, spb;
    sw.fill(0.0f), sb.fill(0.0f), ss.fill(0.0f), spw.fill(0.0f), spb.fill(0.0f);
    for (long i = blockIdx.x; i < items; i += gridDim.x) {
        const Item it = item_rows(a, i);
        Part sg;
        sg.fill(0.0f);
        // Every row group takes the same number of turns: the sums of a row of several waves meet
        // at barriers.
        for (long base = it.first; base < it.end; base += kRows) {
            const bool live = base + sub < it.end;
            const long row = live ? base + sub : it.first;
            const float4 st = reinterpret_cast<const float4*>(stats)[row];
            Part g, t;
            g.load_or(dy, row, D, lane, 0.0f);
            if (a.w) {
                Part w;
                Part n;
                n.load(y, row, D, lane);
                t.load(dh, row, D, lane);
                w.load(a.w, 0, D, lane);
                float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
                for (int e = 0; e < Part::kVals; ++e) {
                    n.v[e] = Part::in(e, lane, D) ? (n.v[e] - st.z) * st.w : 0.0f;
                    if (live) {
                        sb.v[e] += t.v[e];
                        sw.v[e] = fmaf(t.v[e], n.v[e], sw.v[e]);
                    }
                    t.v[e] *= w.v[e];
                    m1 += t.v[e];
                    m2 = fmaf(t.v[e], n.v[e], m2);
                }
                row_sums<LANES>(m1, m2, lds);
                m1 = a.layer ? m1 * inv : 0.0f;
                m2 *= inv;
#pragma unroll
                for (int e = 0; e < Part::kVals; ++e) g.v[e] = fmaf(st.w, t.v[e] - m1 - n.v[e] * m2, g.v[e]);
            }
            if (live) g.store(dx, row, D, lane);
            // t: the unit rows of f (or f), then u
            Part w, b;
            t.load(f, row, D, lane);
            if (a.post_w) {
                w.load(a.post_w, 0, D, lane);
                b.load_or(a.post_b, 0, D, lane, 0.0f);
#pragma unroll
                for (int e = 0; e < Part::kVals; ++e) t.v[e] = Part::in(e, lane, D) ? (t.v[e] - st.x) * st.y : 0.0f;
            }
            Part sc, ga;
            sc.load_or(a.scale, 0, D, lane, 1.0f);
            ga.load_or(a.gate, a.gate_rows ? row : it.image, D, lane, 1.0f);
            float n1 = 0.0f, n2 = 0.0f;
#pragma unroll
            for (int e = 0; e < Part::kVals; ++e) {
                const float u = a.post_w ? fmaf(t.v[e], w.v[e], b.v[e]) : t.v[e];
                const float gu = g.v[e] * u;
                if (live) {
                    ss.v[e] = fmaf(gu, ga.v[e], ss.v[e]);
                    sg.v[e] = fmaf(gu, sc.v[e], sg.v[e]);
                }
                const float du = g.v[e] * (sc.v[e] * ga.v[e]);
                if (a.gate_rows) ga.v[e] = gu * sc.v[e];
                g.v[e] = du;
                if (a.post_w) {
                    if (live) {
                        spb.v[e] += du;
                        spw.v[e] = fmaf(du, t.v[e], spw.v[e]);
                    }
                    g.v[e] = du * w.v[e];
                    n1 += Part::in(e, lane, D) ? g.v[e] : 0.0f;
                    n2 = fmaf(g.v[e], t.v[e], n2);
                }
            }
            if (a.gate_rows && live) ga.store(dgate, row, D, lane);
            if (a.post_w) {
                row_sums<LANES>(n1, n2, lds);
                n1 = a.layer ? n1 * inv : 0.0f;
                n2 *= inv;
#pragma unroll
                for (int e = 0; e < Part::kVals; ++e) g.v[e] = st.y * (g.v[e] - n1 - t.v[e] * n2);
            }
            if (live) g.store(df, row, D, lane);
        }
        if (gate_sums) store_sums<S, LANES, VPL>(sg.v, gate_sums, i, D, lane, sub, lds);
    }
    const long G = gridDim.x, at = blockIdx.x;
    if (a.w) {
        store_sums<S, LANES, VPL>(sw.v, sums, at, D, lane, sub, lds);
        if (a.b) store_sums<S, LANES, VPL>(sb.v, sums, G + at, D, lane, sub, lds);
    }
    if (a.scale) store_sums<S, LANES, VPL>(ss.v, sums, 2 * G + at, D, lane, sub, lds);
    if (a.post_w) {
        store_sums<S, LANES, VPL>(spw.v, sums, 3 * G + at, D, lane, sub, lds);
        if (a.post_b) store_sums<S, LANES, VPL>(spb.v, sums, 4 * G + at, D, lane, sub, lds);
    }
}

struct SumOut {
    void* p[kSums];
};

// out[column] = the groups' sums in order: 16 threads a column take every 16th group, joined in order.
// y > 0 of the grid in sums mode: which sum; in gate mode: which image (its `groups` slots).
__global__ __launch_bounds__(1024) void join_sums_kernel(const float* __restrict__ parts, int groups, int D, int dt,
                                                         SumOut out, void* __restrict__ gate)
{
    constexpr int kCols = 64, kWays = 16;
    __shared__ float lds[kWays][kCols];
    const int col = blockIdx.x * kCols + threadIdx.x % kCols, way = threadIdx.x / kCols;
    const long k = blockIdx.y;
    void* dst = gate ? gate : out.p[k];
    if (dst == nullptr) return;
    float s = 0.0f;
    if (col < D)
        for (int g = way; g < groups; g += kWays) s += parts[(k * groups + g) * D + col];
    lds[way][threadIdx.x % kCols] = s;
    __syncthreads();
    if (way != 0 || col >= D) return;
#pragma unroll
    for (int w = 1; w < kWays; ++w) s += lds[w][threadIdx.x];
    const long at = gate ? k * D + col : col;
    if (dt == kBf16) reinterpret_cast<uint16_t*>(dst)[at] = (uint16_t)f32_to_bf16_rne(s);
    else reinterpret_cast<float*>(dst)[at] = s;
}

// Chunks an image for about `groups` workgroups, each of at least one row a row group.
int chunk_count(const NormCall& a, int groups, int rows)
{
    const long per = std::max(1L, ((long)a.R + a.B - 1) / a.B);
    return (int)std::max(1L, std::min(((long)groups + a.B - 1) / a.B, (per + rows - 1) / rows));
}

// Lanes a row: each lane holds at most 16 values of it (two vectors of bfloat16, four of float32).
template <class S, class F>
hipError_t with_lanes(int D, F&& go)
{
    constexpr int V = S::kBytes == 2 ? 2 : 4;
    const int vpr = D * S::kBytes / 16;
    if (vpr <= 32 * V) return go(std::integral_constant<int, 32>{}, std::integral_constant<int, V>{});
    if (vpr <= 64 * V) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, V>{});
    if (vpr <= 256 * V) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, V>{});
    return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, V>{});
}

template <class S>
hipError_t forward(NormCall a, const void* x, const void* f, void* y, void* h, float* stats, hipStream_t st)
{
    return with_lanes<S>(a.D, [&](auto lanes, auto vpl) {
        constexpr int L = decltype(lanes)::value, V = decltype(vpl)::value;
        a.chunks = chunk_count(a, 4 * kSumGroups, threads<L>() / L);
        hipLaunchKernelGGL((norm_kernel<S, L, V>), dim3((unsigned)((long)a.B * a.chunks)), dim3(threads<L>()), 0, st, a,
                           x, f, y, h, stats);
        return hipGetLastError();
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
        constexpr int L = decltype(lanes)::value, V = decltype(vpl)::value;
        hipLaunchKernelGGL((norm_backward_kernel<S, L, V>), dim3((unsigned)groups), dim3(threads<L>()), 0, st, a, dy, dh,
                           y, f, stats, g.dx, g.df, g.dgate, sums, by_image ? gate_sums : nullptr, items);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    const unsigned cols = (unsigned)((a.D + 63) / 64);
    const SumOut out{{g.dw, g.db, g.dscale, g.dpost_w, g.dpost_b}};
    if (g.dw || g.db || g.dscale || g.dpost_w || g.dpost_b) {
        hipLaunchKernelGGL(join_sums_kernel, dim3(cols, kSums), dim3(1024), 0, st, sums, (int)groups, a.D, a.dt, out,
                           (void*)nullptr);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (by_image) {
        hipLaunchKernelGGL(join_sums_kernel, dim3(cols, (unsigned)a.B), dim3(1024), 0, st, gate_sums, a.chunks, a.D,
                           a.dt, SumOut{}, g.dgate);
        e = hipGetLastError();
    }
    return e;
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

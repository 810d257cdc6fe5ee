// Group norm with an activation over images of rows of C channels, channels last:
//   t = (x - mean) rstd over an image's rows and a group's channels,  z = t w + b,  y = act(z),
// and its gradients, with gz = dy act'(z) and gt = gz w:
//   dx = rstd (gt - mean(gt) - t mean(gt t)),  dw = sum gz t,  db = sum gz.
// A thread keeps one vector of 16 bytes of the channels and walks rows, so that sums are kept by channel
// and groups of any width are sums over channels afterwards.
// Memory bounds it. Slabs of whole groups that fit a workgroup's registers are read once, in one launch; otherwise chunks of
// rows pass twice, with the parts of the sums joined between. 64 grids of 1024 x 768 in bfloat16 with SiLU 45 us, 4.5 TB/s; 16 of
// 4096 x 1024, forward and backward, 199 us, 3.4 TB/s of the 671 MB of one reading and writing each way.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mpm_act.h"
#include "mpm_device.h"
#include "mpm_launch.h"
#include "mpm_work.h"

namespace mpm {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;      // rows a thread loads before it uses them
constexpr int kGroups = 1024;  // workgroups of a pass, about

template <class S>
struct Vec {
    static constexpr int kPer = 16 / S::kBytes;
    u32x4 w;
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (S::kBytes == 2) return e % 2 ? bf16_hi(w[e / 2]) : bf16_lo(w[e / 2]);
        return __uint_as_float(w[e]);
    }
    __device__ static __forceinline__ u32x4 pack(const float (&v)[kPer])
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
};

// How rows and channels are dealt to workgroups: blocks of `cols` vectors of channels, `ways` rows at a time, `chunks`
// parts of an image's rows.
struct Deal {
    int vecs;          // vectors a row
    int cols, ways;    // of a workgroup
    int blocks;        // column blocks (the grid's y)
    int chunks;
    FixedDiv chunks_of;
};

// Rows of an image's chunk: `size` each, the last ones fewer or none.
__device__ __forceinline__ int chunk_size(const Deal& d, long rows)
{
    return rows > 0 ? d.chunks_of((int)(rows - 1)) + 1 : 0;
}

struct Rows {
    long first, end;
    int image;
};
__device__ __forceinline__ Rows image_rows(const GroupNormCall& a, int b)
{
    const long lo = a.off ? a.off[b] : (long)b * a.N, hi = a.off ? a.off[b + 1] : lo + a.N;
    const long first = min(max(lo, 0L), (long)a.R);
    return Rows{first, min(max(hi, first), (long)a.R), b};
}
// The rows of work item i of images x chunks.
__device__ __forceinline__ Rows item_rows(const GroupNormCall& a, const Deal& d, long i)
{
    const int b = d.chunks_of((int)i), c = (int)i - b * d.chunks;
    const Rows r = image_rows(a, b);
    const long size = chunk_size(d, r.end - r.first), first = min(r.first + c * size, r.end);
    return Rows{first, min(first + size, r.end), b};
}

// This thread's vector of channels and its first row's offset (way), if it has any.
struct Place {
    int col, way;
    bool live;
};
__device__ __forceinline__ Place place(const Deal& d)
{
    Place p;
    p.way = threadIdx.x / d.cols;
    p.col = blockIdx.y * d.cols + threadIdx.x % d.cols;
    p.live = p.way < d.ways && p.col < d.vecs;
    return p;
}

// A sum of squares that rounding may have left below zero. (max() would drop a NaN, which an infinity among the values has
// to leave in every value of its group)
template <class F>
__device__ __forceinline__ F not_negative(F v)
{
    return v < 0 ? 0 : v;
}

// Mean and squared deviations of every channel over an item's rows: parts[item][C] pairs, the mean less the channel's value
// in the image's first row, firsts[image][C], so that a mean far from zero beside the deviations costs no digits.
// A thread takes its values from the mean of its own first rows, R: with S and Q the sums of x - R and its square,
// the deviations are Q - S^2 / n. That cancels only as far as R is off the thread's mean, and then those first
// rows themselves deviate as much.
template <class S>
__global__ __launch_bounds__(kThreads) void channel_moments_kernel(GroupNormCall a, Deal d, const uint8_t* x,
                                                                   float2* __restrict__ parts,
                                                                   float* __restrict__ firsts)
{
    typedef Vec<S> V;
    constexpr int kPer = V::kPer;
    __shared__ float2 lds[kPer][kThreads];
    const Rows it = item_rows(a, d, blockIdx.x);
    const Place p = place(d);
    const long stride = (long)a.C * S::kBytes;
    const int rows = (int)(it.end - it.first);
    if (rows == 0) return;
    if (p.live && p.way < rows) {
        const uint8_t* from = x + it.first * stride + (long)p.col * 16;
        const long first = image_rows(a, it.image).first;
        V zero;
        zero.w = load16(x + first * stride + (long)p.col * 16);
        if (it.first == first && p.way == 0) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) firsts[(long)it.image * a.C + p.col * kPer + e] = zero.get(e);
        }
        float ref[kPer], sum[kPer], sq[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) sum[e] = sq[e] = 0.0f;
        for (int row = p.way; row < rows; row += kAhead * d.ways) {
            V v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u].w = load16(from + (long)min(row + u * d.ways, rows - 1) * stride);
            const int n = min(kAhead, (rows - 1 - row) / d.ways + 1);
            if (row == p.way) {
                const float inv = 1.0f / (float)n;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    ref[e] = 0.0f;
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) ref[e] += u < n ? v[u].get(e) - zero.get(e) : 0.0f;
                    ref[e] = fmaf(ref[e], inv, zero.get(e));
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (u >= n) break;
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const float t = v[u].get(e) - ref[e];
                    sum[e] += t;
                    sq[e] = fmaf(t, t, sq[e]);
                }
            }
        }
        const float inv = 1.0f / (float)((rows - 1 - p.way) / d.ways + 1);
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            lds[e][threadIdx.x] = make_float2(fmaf(sum[e], inv, ref[e] - zero.get(e)),
                                              not_negative(fmaf(-sum[e] * inv, sum[e], sq[e])));
    }
    __syncthreads();
    // The threads' parts of each channel, in order.
    const int cols = min(d.cols, d.vecs - (int)blockIdx.y * d.cols), ways = min(d.ways, rows);
    const int whole = rows / d.ways, more = rows - whole * d.ways;  // rows a way: whole, the first `more` one more
    for (int c = threadIdx.x; c < cols * kPer; c += kThreads) {
        const float2* at = lds[c % kPer] + c / kPer;
        float mean = 0.0f, m2 = 0.0f;
        for (int w = 0; w < ways; ++w) mean = fmaf((float)(whole + (w < more)), at[w * d.cols].x, mean);
        mean /= (float)rows;
        for (int w = 0; w < ways; ++w) {
            const float2 q = at[w * d.cols];
            const float e = q.x - mean;
            m2 += fmaf((float)(whole + (w < more)) * e, e, q.y);
        }
        parts[(long)blockIdx.x * a.C + (long)blockIdx.y * d.cols * kPer + c] = make_float2(mean, m2);
    }
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__device__ __forceinline__ float parameter(const void* p, int dt, long i)
{
    if (dt == kBf16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
    return static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_parameter(void* p, int dt, long i, float v)
{
    if (dt == kBf16) static_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_rne(v);
    else static_cast<float*>(p)[i] = v;
}

// What the parts of a channel's rows add to a group's sums, of n (mean - from) and of the squared deviations from it; in 64
// bits, in which the first row's value serves as `from` however far it lies off.
__device__ __forceinline__ double2 spread(float2 part, int n, double offset)
{
    const double u = offset + (double)part.x;
    return make_double2(n * u, (double)part.y + n * u * u);
}

// A group's mean and reciprocal deviation from its sums.
__device__ __forceinline__ float2 finished(const GroupNormCall& a, double count, double from, double2 s)
{
    const double m2 = not_negative(s.y - s.x * s.x / count);
    return make_float2((float)(from + s.x / count), (float)(1.0 / sqrt(m2 / count + (double)a.eps)));
}

constexpr int kJoinThreads = 1024;
// The sums of two numbers of each of `many` items over a workgroup of kJoinThreads, in a fixed order, in every thread.
template <class Use>
__device__ __forceinline__ double2 block_sum(int many, Use&& use)
{
    __shared__ double2 lds[kJoinThreads / kWave];
    double s = 0.0, s2 = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x; i < many; i += kJoinThreads) {
        const double2 q = use(i);
        s += q.x;
        s2 += q.y;
    }
    s = wave_sum(s);
    s2 = wave_sum(s2);
    __syncthreads();  // the sums before have been read
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = make_double2(s, s2);
    __syncthreads();
    double2 r = lds[0];
    for (int w = 1; w < kJoinThreads / kWave; ++w) {
        r.x += lds[w].x;
        r.y += lds[w].y;
    }
    return r;
}

// A channel's parts of an image joined over its chunks, 16 channels a workgroup, 64 shares of the chunks each joined by a wave:
// what enters its group's sums. firsts: the parts are moments (spread), otherwise sums.
constexpr int kJoinWaves = kJoinThreads / kWave;
__global__ __launch_bounds__(kJoinThreads) void join_chunks_kernel(GroupNormCall a, Deal d, const float2* __restrict__ parts,
                                                                   const float* __restrict__ firsts,
                                                                   double2* __restrict__ joined)
{
    __shared__ double2 lds[kWave][kJoinWaves + 1];
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, local = t % kJoinWaves, way = t / kJoinWaves;
    const int c0 = blockIdx.x * kJoinWaves, c = min(c0 + local, a.C - 1), width = a.C / a.groups;
    for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
        const Rows image = image_rows(a, b);
        const int rows = (int)(image.end - image.first), size = chunk_size(d, rows);
        const int chunks = !firsts ? d.chunks : rows > 0 ? (rows - 1) / size + 1 : 0;
        double2 s = make_double2(0.0, 0.0);
        const float* f = firsts ? firsts + (long)b * a.C : nullptr;
        const double offset = firsts && rows > 0 ? (double)f[c] - (double)f[c / width * width] : 0.0;
        const float2* at = parts + (long)b * d.chunks * a.C + c;
#pragma unroll 4
        for (int k = way; k < chunks; k += kWave) {
            const float2 p = at[(long)k * a.C];
            const double2 q = firsts ? spread(p, min(size, rows - k * size), offset) : make_double2((double)p.x, (double)p.y);
            s.x += q.x;
            s.y += q.y;
        }
        __syncthreads();  // the image before has been read
        lds[way][local] = s;
        __syncthreads();
        const double2 own = lds[lane][wave];
        s = make_double2(wave_sum(own.x), wave_sum(own.y));
        if (lane == 0 && c0 + wave < a.C) joined[(long)b * a.C + c0 + wave] = s;
    }
}

// Mean and reciprocal deviation of every image and group, a workgroup each; from the channels' joined parts where they are
// given.
__global__ __launch_bounds__(kJoinThreads) void group_stats_kernel(GroupNormCall a, Deal d, FixedDiv width_of,
                                                               const float2* __restrict__ parts,
                                                               const double2* __restrict__ joined,
                                                               const float* __restrict__ firsts,
                                                               float2* __restrict__ stats)
{
    const int width = a.C / a.groups;
    for (long pair = blockIdx.x; pair < (long)a.B * a.groups; pair += gridDim.x) {
        const int b = (int)(pair / a.groups), g = (int)(pair % a.groups);
        const Rows image = image_rows(a, b);
        const int rows = (int)(image.end - image.first), size = chunk_size(d, rows);
        const float* f = firsts + (long)b * a.C + g * width;
        const float2* at = parts + (long)b * d.chunks * a.C + g * width;
        const double from = rows > 0 ? (double)f[0] : 0.0;
        const int chunks = rows > 0 ? (rows - 1) / size + 1 : 0;  // that have rows
        const double2 s = joined ? block_sum(rows > 0 ? width : 0, [&](int i) { return joined[(long)b * a.C + g * width + i]; })
                                 : block_sum(chunks * width, [&](int i) {
                                       const int k = width_of(i), c = i - k * width;
                                       return spread(at[(long)k * a.C + c], min(size, rows - k * size), (double)f[c] - from);
                                   });
        if (threadIdx.x == 0)
            stats[pair] = rows > 0 ? finished(a, (double)rows * width, from, s) : make_float2(0.0f, 0.0f);
    }
}

// The groups that a column block's channels belong to.
struct GroupRange {
    int first, count;
};
template <class S>
__device__ __forceinline__ GroupRange block_groups(const GroupNormCall& a, const Deal& d)
{
    const int width = a.C / a.groups, c0 = blockIdx.y * d.cols * Vec<S>::kPer;
    const int c1 = min(c0 + d.cols * Vec<S>::kPer, a.C) - 1;
    return GroupRange{c0 / width, c1 / width - c0 / width + 1};
}
// Channels of them that a workgroup joins by itself, at most.
constexpr int kMostChannels = kThreads * 8;

// Sums over the channels of each of a block's groups, `lanes` lanes a group (8 for many groups: 32 of 6 channels 11.5 us, with
// 64 lanes 17.6): use(channel of the block's groups) gives two numbers, write(group, sums) takes their sums.
template <class Use, class Write>
__device__ __forceinline__ void over_channels(int groups, int width, Use&& use, Write&& write)
{
    const int lanes = groups <= 8 ? kWave : 8;
    const int lane = threadIdx.x % lanes;
    for (int g = threadIdx.x / lanes; g < groups; g += kThreads / lanes) {
        double s = 0.0, s2 = 0.0;
        for (int c = lane; c < width; c += lanes) {
            const double2 q = use(g * width + c);
            s += q.x;
            s2 += q.y;
        }
        for (int o = lanes / 2; o > 0; o >>= 1) {
            s += __shfl_xor(s, o);
            s2 += __shfl_xor(s2, o);
        }
        if (lane == 0) write(g, make_double2(s, s2));
    }
}

// A vector's parameters: mean, rstd, weight and shift of each of its channels.
template <class S>
struct Affine {
    static constexpr int kPer = Vec<S>::kPer;
    float mean[kPer], rstd[kPer], w[kPer], b[kPer];

    // stats: of groups from `first` on.
    __device__ __forceinline__ void load(const GroupNormCall& a, const float2* stats, int first, int col)
    {
        Vec<S> wv, bv;
        if (a.w) wv.w = load16(static_cast<const uint8_t*>(a.w) + col * 16);
        if (a.b) bv.w = load16(static_cast<const uint8_t*>(a.b) + col * 16);
        const int width = a.C / a.groups;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float2 s = stats[(col * kPer + e) / width - first];
            mean[e] = s.x;
            rstd[e] = s.y;
            w[e] = a.w ? wv.get(e) : 1.0f;
            b[e] = a.b ? bv.get(e) : 0.0f;
        }
    }
};

// y from x and the statistics: stats where they are given, otherwise from the parts (of few items), in every workgroup by
// itself, and written to `made` (may be null).
template <class S, int ACT>
__global__ __launch_bounds__(kThreads) void apply_kernel(GroupNormCall a, Deal d, const uint8_t* x, uint8_t* y,
                                                         const float2* __restrict__ stats,
                                                         const float2* __restrict__ parts,
                                                         const float* __restrict__ firsts, float2* __restrict__ made)
{
    typedef Vec<S> V;
    __shared__ float2 own[kMostChannels];
    __shared__ double2 sums[kMostChannels];
    const Rows it = item_rows(a, d, blockIdx.x);
    const Place p = place(d);
    const GroupRange groups = block_groups<S>(a, d);
    if (!stats) {
        const Rows image = image_rows(a, it.image);
        const int rows = (int)(image.end - image.first), width = a.C / a.groups, c0 = groups.first * width;
        const float* f = firsts + (long)it.image * a.C + c0;
        const int size = chunk_size(d, rows), chunks = rows > 0 ? (rows - 1) / size + 1 : 0;
        for (int c = threadIdx.x; rows > 0 && c < groups.count * width; c += kThreads) {
            const float2* at = parts + (long)it.image * d.chunks * a.C + c0 + c;
            const double offset = (double)f[c] - (double)f[c / width * width];
            double s = 0.0, s2 = 0.0;
#pragma unroll 8
            for (int k = 0; k < chunks; ++k) {
                const double2 q = spread(at[(long)k * a.C], min(size, rows - k * size), offset);
                s += q.x;
                s2 += q.y;
            }
            sums[c] = make_double2(s, s2);
        }
        __syncthreads();
        over_channels(
            groups.count, width, [&](int c) { return rows > 0 ? sums[c] : make_double2(0.0, 0.0); },
            [&](int g, double2 s) {
                const float2 q = rows > 0 ? finished(a, (double)rows * width, (double)f[g * width], s) : make_float2(0.0f, 0.0f);
                own[g] = q;
                // (a group that two column blocks share gets the same value from both)
                if (made && it.first == image.first) made[(long)it.image * a.groups + groups.first + g] = q;
            });
        __syncthreads();
    }
    if (!p.live || it.first >= it.end) return;
    const long stride = (long)a.C * S::kBytes;
    Affine<S> f;
    if (stats) f.load(a, stats + (long)it.image * a.groups, 0, p.col);
    else f.load(a, own, groups.first, p.col);
    for (long row = it.first + p.way; row < it.end; row += kAhead * d.ways) {
        V v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (row + u * d.ways < it.end) v[u].w = load16(x + (row + u * d.ways) * stride + p.col * 16);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const long r = row + u * d.ways;
            if (r >= it.end) break;
            float o[V::kPer];
#pragma unroll
            for (int e = 0; e < V::kPer; ++e)
                o[e] = activate<ACT, S::kBytes == 4>(fmaf((v[u].get(e) - f.mean[e]) * f.rstd[e], f.w[e], f.b[e]));
            store16_stream(y + r * stride + p.col * 16, V::pack(o));
        }
    }
}

// The sums of gz and gz t of every channel over an item's rows: parts[item][C] pairs.
template <class S, int ACT>
__global__ __launch_bounds__(kThreads) void channel_sums_kernel(GroupNormCall a, Deal d, const uint8_t* dy,
                                                                const uint8_t* x, const float2* __restrict__ stats,
                                                                float2* __restrict__ parts)
{
    typedef Vec<S> V;
    __shared__ float2 lds[kThreads];
    const Rows it = item_rows(a, d, blockIdx.x);
    const Place p = place(d);
    const long stride = (long)a.C * S::kBytes;
    float s0[V::kPer], s1[V::kPer];
#pragma unroll
    for (int e = 0; e < V::kPer; ++e) s0[e] = s1[e] = 0.0f;
    if (p.live && it.first < it.end) {
        Affine<S> f;
        f.load(a, stats + (long)it.image * a.groups, 0, p.col);
        for (long row = it.first + p.way; row < it.end; row += kAhead * d.ways) {
            V v[kAhead], g[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const long r = row + u * d.ways;
                if (r < it.end) {
                    v[u].w = load16(x + r * stride + p.col * 16);
                    g[u].w = load16(dy + r * stride + p.col * 16);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (row + u * d.ways >= it.end) break;
#pragma unroll
                for (int e = 0; e < V::kPer; ++e) {
                    const float t = (v[u].get(e) - f.mean[e]) * f.rstd[e];
                    const float gz = g[u].get(e) * activation_slope<ACT, S::kBytes == 4>(fmaf(t, f.w[e], f.b[e]));
                    s0[e] += gz;
                    s1[e] = fmaf(gz, t, s1[e]);
                }
            }
        }
    }
    for (int e = 0; e < V::kPer; ++e) {
        __syncthreads();
        lds[threadIdx.x] = make_float2(s0[e], s1[e]);
        __syncthreads();
        if (p.live && p.way == 0) {
            float2 q = lds[threadIdx.x];
            for (int w = 1; w < d.ways; ++w) {
                q.x += lds[w * d.cols + threadIdx.x].x;
                q.y += lds[w * d.cols + threadIdx.x].y;
            }
            parts[(long)blockIdx.x * a.C + p.col * V::kPer + e] = q;
        }
    }
}

// A channel's sums as they enter its group's: of gt and gt t.
__device__ __forceinline__ double2 weighted(const GroupNormCall& a, double2 q, int c)
{
    const double w = a.w ? (double)parameter(a.w, a.dt, c) : 1.0;
    return make_double2(w * q.x, w * q.y);
}

// From the channels' sums: the means of gt and gt t of every image and group, a workgroup each ...
__global__ __launch_bounds__(kJoinThreads) void group_means_kernel(GroupNormCall a, Deal d, FixedDiv width_of,
                                                               const float2* __restrict__ parts,
                                                               const double2* __restrict__ joined,
                                                               float2* __restrict__ means)
{
    const int width = a.C / a.groups;
    for (long pair = blockIdx.x; pair < (long)a.B * a.groups; pair += gridDim.x) {
        const int b = (int)(pair / a.groups), g = (int)(pair % a.groups);
        const float2* at = parts + (long)b * d.chunks * a.C + g * width;
        const double2 s = joined ? block_sum(width, [&](int i) {
            return weighted(a, joined[(long)b * a.C + g * width + i], g * width + i);
        }) : block_sum(d.chunks * width, [&](int i) {
            const int k = width_of(i), c = i - k * width;
            const float2 q = at[(long)k * a.C + c];
            return weighted(a, make_double2((double)q.x, (double)q.y), g * width + c);
        });
        const Rows r = image_rows(a, b);
        const double n = (double)(r.end - r.first) * width;
        if (threadIdx.x == 0)
            means[pair] = n > 0.0 ? make_float2((float)(s.x / n), (float)(s.y / n)) : make_float2(0.0f, 0.0f);
    }
}

// ... and dw and db, 64 channels a workgroup, sixteen waves' shares of the items joined in order.
__global__ __launch_bounds__(kJoinThreads) void join_sums_kernel(const float2* __restrict__ parts, long items, int C,
                                                                      int dt, void* dw, void* db)
{
    __shared__ double lds[2][kJoinWaves][kWave];
    const int lane = threadIdx.x % kWave, way = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    double s0 = 0.0, s1 = 0.0;
    if (c < C) {
#pragma unroll 4
        for (long i = way; i < items; i += kJoinWaves) {
            const float2 q = parts[i * C + c];
            s0 += (double)q.x;
            s1 += (double)q.y;
        }
    }
    lds[0][way][lane] = s0;
    lds[1][way][lane] = s1;
    __syncthreads();
    if (way != 0 || c >= C) return;
    for (int w = 1; w < kJoinWaves; ++w) {
        s0 += lds[0][w][lane];
        s1 += lds[1][w][lane];
    }
    if (db) store_parameter(db, dt, c, (float)s0);
    if (dw) store_parameter(dw, dt, c, (float)s1);
}

// dx, from the means where they are given, otherwise from the parts, as apply_kernel.
template <class S, int ACT>
__global__ __launch_bounds__(kThreads) void input_gradient_kernel(GroupNormCall a, Deal d, const uint8_t* dy,
                                                                  const uint8_t* x, uint8_t* dx,
                                                                  const float2* __restrict__ stats,
                                                                  const float2* __restrict__ means,
                                                                  const float2* __restrict__ parts)
{
    typedef Vec<S> V;
    __shared__ float2 own[kMostChannels];
    __shared__ double2 sums[kMostChannels];
    const Place p = place(d);
    const Rows it = item_rows(a, d, blockIdx.x);
    const GroupRange groups = block_groups<S>(a, d);
    if (!means) {
        const Rows image = image_rows(a, it.image);
        const int width = a.C / a.groups, c0 = groups.first * width;
        const double n = (double)(image.end - image.first) * width;
        for (int c = threadIdx.x; c < groups.count * width; c += kThreads) {
            const float2* at = parts + (long)it.image * d.chunks * a.C + c0 + c;
            double s0 = 0.0, s1 = 0.0;
#pragma unroll 8
            for (int k = 0; k < d.chunks; ++k) {
                const float2 q = at[(long)k * a.C];
                s0 += (double)q.x;
                s1 += (double)q.y;
            }
            sums[c] = weighted(a, make_double2(s0, s1), c0 + c);
        }
        __syncthreads();
        over_channels(
            groups.count, width, [&](int c) { return sums[c]; },
            [&](int g, double2 s) {
                own[g] = n > 0.0 ? make_float2((float)(s.x / n), (float)(s.y / n)) : make_float2(0.0f, 0.0f);
            });
        __syncthreads();
    }
    if (!p.live) return;
    const long stride = (long)a.C * S::kBytes;
    if (a.off) {  // a share of the rows of no image
        const u32x4 none = {0, 0, 0, 0};
        const long lo = min(max((long)a.off[0], 0L), (long)a.R), hi = min(max((long)a.off[a.B], lo), (long)a.R);
        const long many = lo + a.R - hi, first = many * blockIdx.x / gridDim.x, end = many * (blockIdx.x + 1L) / gridDim.x;
        for (long r = first + p.way; r < end; r += d.ways)
            store16(dx + (r < lo ? r : r - lo + hi) * stride + p.col * 16, none);
    }
    if (it.first >= it.end) return;
    Affine<S> f;
    f.load(a, stats + (long)it.image * a.groups, 0, p.col);
    float m0[V::kPer], m1[V::kPer];
#pragma unroll
    for (int e = 0; e < V::kPer; ++e) {
        const int g = (p.col * V::kPer + e) / (a.C / a.groups);
        const float2 m = means ? means[(long)it.image * a.groups + g] : own[g - groups.first];
        m0[e] = m.x;
        m1[e] = m.y;
    }
    for (long row = it.first + p.way; row < it.end; row += kAhead * d.ways) {
        V v[kAhead], g[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const long r = row + u * d.ways;
            if (r < it.end) {
                v[u].w = load16(x + r * stride + p.col * 16);
                g[u].w = load16(dy + r * stride + p.col * 16);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const long r = row + u * d.ways;
            if (r >= it.end) break;
            float o[V::kPer];
#pragma unroll
            for (int e = 0; e < V::kPer; ++e) {
                const float t = (v[u].get(e) - f.mean[e]) * f.rstd[e];
                const float gz = g[u].get(e) * activation_slope<ACT, S::kBytes == 4>(fmaf(t, f.w[e], f.b[e]));
                o[e] = f.rstd[e] * (fmaf(gz, f.w[e], -m0[e]) - t * m1[e]);
            }
            store16_stream(dx + r * stride + p.col * 16, V::pack(o));
        }
    }
}

// ---- images whose part of some groups stays in registers ---------------------------------
//
// A workgroup takes a slab of whole groups of one image: it reads the slab once, keeps it, and writes it. Rows past what
// its registers hold are read again (the host picks slabs that fit, but for packed images it knows only their
// average).

constexpr int kSlabThreads = 1024;

struct Slab {
    int vecs, cols, slabs, ways, threads;
    int width;       // channels a group
    int groups;      // of a slab
    bool stream;     // whether its rows are whole lines, or many, and written past the L2
    FixedDiv cols_of, width_of, per_of;  // by cols; by a group's channels; by its vectors (where it has whole ones)
};

// Rows of whole lines written past the L2, whose room the slabs' reads need (64 grids of 1024 x 768 51.6 -> 48 us, a step
// of 16 of 4096 x 1024 219 -> 197); parts of lines by way of it, which joins them (4 of 9216 x 256, 16 bytes a slab: 24 us
// against 51).
__device__ __forceinline__ void store_piece(uint8_t* p, u32x4 v, bool stream)
{
    if (stream) {
        store16_stream(p, v);
    } else {
        asm volatile("" ::: "memory");  // (the compiler would make one store of the two, an ordinary one,
        store16(p, v);
        asm volatile("" ::: "memory");  // before the branch or behind it)
    }
}

// Slab and image of a workgroup: the slabs of an image on one XCD, whose L2 then joins the lines that two of them share.
constexpr int kXcds = 8;
__device__ __forceinline__ bool slab_item(long items, long* item)
{
    const int xcd = blockIdx.x % kXcds;
    *item = items * xcd / kXcds + blockIdx.x / kXcds;
    return *item < items * (xcd + 1) / kXcds;
}

constexpr int kMostSlabGroups = 256;

// The sums of N values of every thread over each group of the slab, in LDS out[n][group]. v: by channel of the thread's
// vector; ONE: a vector lies in one group.
template <class S, bool ONE, int N>
__device__ __forceinline__ void group_sums(const float (&v)[N][Vec<S>::kPer], const Slab& s, float* lds,
                                           float (*out)[kMostSlabGroups])
{
    constexpr int kPer = Vec<S>::kPer, kValue = (ONE ? 1 : kPer) * kSlabThreads;  // numbers in LDS of a value
    const int t = threadIdx.x, lane = t % kWave;
    __syncthreads();  // what was in LDS has been read
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if constexpr (ONE) {
            float one = 0.0f;
#pragma unroll
            for (int e = 0; e < kPer; ++e) one += v[n][e];
            lds[n * kValue + t] = one;
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e) lds[n * kValue + e * kSlabThreads + t] = v[n][e];
        }
    }
    __syncthreads();
    const int per = ONE ? s.width / kPer : s.width, many = per * s.ways;
    for (int g = t / kWave; g < s.groups; g += s.threads / kWave) {
        float sum[N] = {};
        for (int i = lane; i < many; i += kWave) {
            const int way = ONE ? s.per_of(i) : s.width_of(i), c = g * per + i - way * per;
            if (!ONE && c >= s.cols * kPer) continue;
            const float* at = lds + (ONE ? way * s.cols + c : c % kPer * kSlabThreads + way * s.cols + c / kPer);
#pragma unroll
            for (int n = 0; n < N; ++n) sum[n] += at[n * kValue];
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float all = lanes_sum<kWave>(sum[n]);
            if (lane == 0) out[n][g] = all;
        }
    }
    __syncthreads();
}

// Group g of the slab that channel e of this thread's vector belongs to.
template <class S, bool ONE>
__device__ __forceinline__ int slab_group(const Slab& s, int col, int e)
{
    constexpr int kPer = Vec<S>::kPer;
    return ONE ? s.per_of(col) : s.width_of(col * kPer + e);
}

template <class S, int ACT, bool ONE, int VPT>
__global__ __launch_bounds__(kSlabThreads) void slab_kernel(GroupNormCall a, Slab s, const uint8_t* x, uint8_t* y,
                                                            float2* __restrict__ stats)
{
    typedef Vec<S> V;
    constexpr int kPer = V::kPer, kOwn = ONE ? 1 : kPer;  // statistics a vector has
    // A group's mean is that of its values less its first one, which leaves a mean far from zero its digits; its
    // deviations are taken from the mean. A first value far off costs that mean up to half its distance's step (2^-24), which
    // float32 results would show: there the deviations' own mean corrects it (7 images of 670 x 836, 11 groups: 12.9 -> 13.4
    // us, 1 of 1024 x 192, 32 groups 12.6 -> 14.7), while bfloat16 rounds 2^16 times as coarsely.
    constexpr int kSums = S::kBytes == 4 ? 2 : 1;  // squared deviations and, in float32, deviations
    __shared__ float lds[kSums * (ONE ? 1 : kPer) * kSlabThreads];
    __shared__ float sums[kSums][kMostSlabGroups];
    long item;
    if (!slab_item((long)a.B * s.slabs, &item)) return;
    const int b = (int)(item / s.slabs), slab = (int)(item % s.slabs);
    const Rows it = image_rows(a, b);
    const int n = (int)(it.end - it.first), t = threadIdx.x, way = s.cols_of(t), local = t - way * s.cols;
    const int col = slab * s.cols + local, groups = min(s.groups, a.groups - slab * s.groups);
    const bool live = way < s.ways && col < s.vecs;
    float2* out = stats ? stats + (long)b * a.groups + slab * s.groups : nullptr;
    if (n == 0) {
        if (out && t < groups) out[t] = make_float2(0.0f, 0.0f);
        return;
    }
    const long stride = (long)a.C * S::kBytes;
    const uint8_t* from = x + it.first * stride + (long)col * 16;
    V v[VPT];
    const u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
        const int r = way + u * s.ways;
        v[u].w = none;
        if (live && r < n) v[u].w = load16(from + r * stride);
    }
    const int rest = way + VPT * s.ways;  // the first row that is not kept
    float first[kOwn], mean[kOwn], rstd[kOwn];
    int group[kOwn];
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        group[e] = live ? slab_group<S, ONE>(s, local, e) : 0;
        first[e] = parameter(x, a.dt, it.first * a.C + (long)(slab * s.groups + group[e]) * s.width);
    }
    const float count = (float)n * (float)s.width;
    auto each = [&](auto&& use) {  // every value of the thread's rows and channels
#pragma unroll
        for (int u = 0; u < VPT; ++u)
            if (live && way + u * s.ways < n) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) use(v[u].get(e), e);
            }
        if (live)
            for (int r = rest; r < n; r += s.ways) {
                V w;
                w.w = load16(from + r * stride);
#pragma unroll
                for (int e = 0; e < kPer; ++e) use(w.get(e), e);
            }
    };
    float one[1][kPer] = {}, two[kSums][kPer] = {};
    each([&](float f, int e) { one[0][e] += f - first[ONE ? 0 : e]; });
    group_sums<S, ONE>(one, s, lds, sums);
#pragma unroll
    for (int e = 0; e < kOwn; ++e) mean[e] = first[e] + sums[0][group[e]] / count;
    each([&](float f, int e) {
        const float d = f - mean[ONE ? 0 : e];
        two[0][e] = fmaf(d, d, two[0][e]);
        if constexpr (kSums > 1) two[1][e] += d;
    });
    group_sums<S, ONE>(two, s, lds, sums);
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        float var = sums[0][group[e]] / count;
        if constexpr (kSums > 1) {
            const float by = sums[1][group[e]] / count;
            mean[e] += by;
            var = not_negative(fmaf(-by, by, var));
        }
        rstd[e] = 1.0f / sqrtf(var + a.eps);
    }
    if (!live) return;
    // (a thread of each group's first channel has its statistics)
    if (out && way == 0) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int c = local * kPer + e, g = group[ONE ? 0 : e];
            if (c == g * s.width && g < groups) out[g] = make_float2(mean[ONE ? 0 : e], rstd[ONE ? 0 : e]);
        }
    }
    V wv, bv;
    if (a.w) wv.w = load16(static_cast<const uint8_t*>(a.w) + col * 16);
    if (a.b) bv.w = load16(static_cast<const uint8_t*>(a.b) + col * 16);
    auto write = [&](const V& f, int r) {
        float o[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            o[e] = activate<ACT, S::kBytes == 4>(fmaf((f.get(e) - mean[ONE ? 0 : e]) * rstd[ONE ? 0 : e],
                                                      a.w ? wv.get(e) : 1.0f, a.b ? bv.get(e) : 0.0f));
        store_piece(y + it.first * stride + (long)col * 16 + r * stride, V::pack(o), s.stream);
    };
#pragma unroll
    for (int u = 0; u < VPT; ++u)
        if (way + u * s.ways < n) write(v[u], way + u * s.ways);
    for (int r = rest; r < n; r += s.ways) {
        V w;
        w.w = load16(from + r * stride);
        write(w, r);
    }
}

// The gradients likewise: the slab of x and dy kept between the sums and dx. parts[image][C]: the channels' sums of gz and
// gz t, for dw and db.
template <class S, int ACT, bool ONE, int VPT>
__global__ __launch_bounds__(kSlabThreads) void slab_backward_kernel(GroupNormCall a, Slab s, const uint8_t* dy,
                                                                     const uint8_t* x, uint8_t* dx,
                                                                     const float2* __restrict__ stats,
                                                                     float2* __restrict__ parts)
{
    typedef Vec<S> V;
    constexpr int kPer = V::kPer, kOwn = ONE ? 1 : kPer;
    __shared__ float lds[kPer * kSlabThreads];
    __shared__ float sums[2][kMostSlabGroups];
    const long items = (long)a.B * s.slabs;
    long item;
    if (!slab_item(items, &item)) return;
    const int b = (int)(item / s.slabs), slab = (int)(item % s.slabs);
    const Rows it = image_rows(a, b);
    const int n = (int)(it.end - it.first), t = threadIdx.x, way = s.cols_of(t), local = t - way * s.cols;
    const int col = slab * s.cols + local;
    const bool live = way < s.ways && col < s.vecs;
    const long stride = (long)a.C * S::kBytes;
    if (a.off && live) {  // a share of the rows of no image
        const u32x4 none = {0, 0, 0, 0};
        const long lo = min(max((long)a.off[0], 0L), (long)a.R), hi = min(max((long)a.off[a.B], lo), (long)a.R);
        const long many = lo + a.R - hi, end = many * (b + 1L) / a.B;
        for (long r = many * b / a.B + way; r < end; r += s.ways)
            store16(dx + (r < lo ? r : r - lo + hi) * stride + (long)col * 16, none);
    }
    const long at = it.first * stride + (long)col * 16;
    V v[VPT], g[VPT];
    const u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
        const int r = way + u * s.ways;
        v[u].w = g[u].w = none;
        if (live && r < n) {
            v[u].w = load16(x + at + r * stride);
            g[u].w = load16(dy + at + r * stride);
        }
    }
    const int rest = way + VPT * s.ways;
    V wv, bv;
    wv.w = bv.w = none;
    if (a.w && live) wv.w = load16(static_cast<const uint8_t*>(a.w) + col * 16);
    if (a.b && live) bv.w = load16(static_cast<const uint8_t*>(a.b) + col * 16);
    float mean[kOwn], rstd[kOwn], s0[kPer], s1[kPer];
    int group[kOwn];
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        group[e] = live ? slab_group<S, ONE>(s, local, e) : 0;
        const float2 q = stats[(long)b * a.groups + slab * s.groups + group[e]];
        mean[e] = q.x;
        rstd[e] = q.y;
    }
    auto weight = [&](int e) { return a.w ? wv.get(e) : 1.0f; };
    // t and gz of a value and its gradient.
    auto slope = [&](float f, float d, int e, float* gz) {
        const float u = (f - mean[ONE ? 0 : e]) * rstd[ONE ? 0 : e];
        *gz = d * activation_slope<ACT, S::kBytes == 4>(fmaf(u, weight(e), a.b ? bv.get(e) : 0.0f));
        return u;
    };
#pragma unroll
    for (int e = 0; e < kPer; ++e) s0[e] = s1[e] = 0.0f;
    auto add = [&](const V& f, const V& d) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            float gz;
            const float u = slope(f.get(e), d.get(e), e, &gz);
            s0[e] += gz;
            s1[e] = fmaf(gz, u, s1[e]);
        }
    };
#pragma unroll
    for (int u = 0; u < VPT; ++u)
        if (live && way + u * s.ways < n) add(v[u], g[u]);
    if (live)
        for (int r = rest; r < n; r += s.ways) {
            V f, d;
            f.w = load16(x + at + r * stride);
            d.w = load16(dy + at + r * stride);
            add(f, d);
        }
    // The channels' sums, for dw and db, one value of every thread's vector at a time ...
    if (parts) {
        const int lane = t % kWave, channels = min(s.cols, s.vecs - slab * s.cols) * kPer;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kPer; ++e) lds[e * kSlabThreads + t] = k ? s1[e] : s0[e];
            __syncthreads();
            for (int c = t / kWave; c < channels; c += s.threads / kWave) {
                const float* p = lds + c % kPer * kSlabThreads + c / kPer;
                float sum = 0.0f;
                for (int w = lane; w < s.ways; w += kWave) sum += p[w * s.cols];
                sum = lanes_sum<kWave>(sum);
                if (lane == 0)
                    reinterpret_cast<float*>(parts)[2 * ((long)b * a.C + (long)slab * s.cols * kPer + c) + k] = sum;
            }
        }
    }
    // ... and the groups', of gt and gt t.
    float gt[1][kPer], gtt[1][kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        gt[0][e] = s0[e] * weight(e);
        gtt[0][e] = s1[e] * weight(e);
    }
    group_sums<S, ONE>(gt, s, lds, sums);
    group_sums<S, ONE>(gtt, s, lds, sums + 1);
    if (!live) return;
    const float inv = 1.0f / ((float)n * (float)s.width);
    float m0[kOwn], m1[kOwn];
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        m0[e] = sums[0][group[e]] * inv;
        m1[e] = sums[1][group[e]] * inv;
    }
    auto write = [&](const V& f, const V& d, int r) {
        float o[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            float gz;
            const float u = slope(f.get(e), d.get(e), e, &gz);
            o[e] = rstd[ONE ? 0 : e] * (fmaf(gz, weight(e), -m0[ONE ? 0 : e]) - u * m1[ONE ? 0 : e]);
        }
        store_piece(dx + at + r * stride, V::pack(o), s.stream);
    };
#pragma unroll
    for (int u = 0; u < VPT; ++u)
        if (way + u * s.ways < n) write(v[u], g[u], way + u * s.ways);
    for (int r = rest; r < n; r += s.ways) {
        V f, d;
        f.w = load16(x + at + r * stride);
        d.w = load16(dy + at + r * stride);
        write(f, d, r);
    }
}

// How a call goes by slabs: `vpt` vectors a thread keeps of a tensor, for images of the average length. Slabs are the
// widest whole groups that fit and leave a workgroup for every compute unit, of whole 64-byte pieces where groups allow;
// vecs of a slab 0: no slab fits.
struct Plan {
    Slab s;
    int vpt;
};
constexpr int kUnits = 256;

int common_divisor(int a, int b) { return b ? common_divisor(b, a % b) : a; }

Plan plan(const GroupNormCall& a, bool backward)
{
    const int bytes = a.dt == kBf16 ? 2 : 4, per = 16 / bytes, width = a.C / a.groups;
    const int unit = width / common_divisor(width, per);   // vectors of the fewest whole groups that fill vectors
    const int unit_groups = unit * per / width;
    const int vecs = a.C / per, units = vecs / unit;
    const long rows = std::max(1L, ((long)a.R + a.B - 1) / a.B);
    const int most = backward ? 8 : 16;
    int best = 0;
    double best_use = 0.0;
    for (int k = 1; k <= units; ++k) {
        const int cols = unit * k;
        if (cols > kSlabThreads / 4 || (long)unit_groups * k > kMostSlabGroups) break;
        const bool fits = (kSlabThreads / cols) * (long)most >= rows;
        const long groups = (long)a.B * ((units + k - 1) / k);
        if (k > 1 && (!fits || groups < kUnits)) break;
        const int len = cols * 16;
        const double use = len % 128 == 0 || k == units ? 1.0 : (double)len / (len + 128 - common_divisor(len, 128));
        if (use > best_use + 0.05) {
            best_use = use;
            best = k;
        }
    }
    Plan p{Slab{vecs, 0, 0, 0, 0, width, 0, false, FixedDiv(1), FixedDiv((uint32_t)width), FixedDiv((uint32_t)std::max(1, width / per))},
           1};
    if (best == 0) return p;
    Slab& s = p.s;
    s.cols = unit * best;
    s.slabs = (units + best - 1) / best;
    s.groups = unit_groups * best;
    s.cols_of = FixedDiv((uint32_t)s.cols);
    s.stream = s.cols % 4 == 0 || s.cols >= 6 || s.slabs == 1;
    // Enough threads for about four vectors each.
    s.threads = kSlabThreads;
    while (s.threads > 256 && s.cols * 2 <= s.threads / 4 && (s.threads / 2 / s.cols) * 4L >= rows) s.threads /= 2;
    s.ways = s.threads / s.cols;
    p.vpt = rows <= (long)s.ways * (most / 4) ? most / 4 : most;
    return p;
}

Deal deal(const GroupNormCall& a)
{
    Deal d{0, 0, 0, 0, 0, FixedDiv(1)};
    d.vecs = a.C / (a.dt == kBf16 ? 8 : 4);
    // Few enough vectors for two rows at a time; blocks of about the same width.
    d.blocks = (d.vecs + kThreads - 1) / kThreads;
    d.cols = (d.vecs + d.blocks - 1) / d.blocks;
    d.ways = kThreads / d.cols;
    const long per = std::max(1L, ((long)a.R + a.B - 1) / a.B);
    const long most = std::max(1L, (per + d.ways * kAhead - 1) / (d.ways * kAhead));
    d.chunks = (int)std::max(1L, std::min(most, ((long)kGroups / d.blocks + a.B - 1) / a.B));
    d.chunks_of = FixedDiv((uint32_t)d.chunks);
    return d;
}

// Workgroups for the images' groups (which may be more than a grid has).
unsigned pair_groups(const GroupNormCall& a) { return (unsigned)std::min((long)a.B * a.groups, 1L << 18); }

size_t aligned256(size_t v) { return (v + 255) / 256 * 256; }
size_t parts_bytes(const GroupNormCall& a, const Deal& d) { return aligned256((size_t)a.B * d.chunks * a.C * 8); }
size_t firsts_bytes(const GroupNormCall& a) { return aligned256((size_t)a.B * a.C * 4); }
size_t stats_bytes(const GroupNormCall& a) { return aligned256((size_t)a.B * a.groups * 8); }

// Whether the second pass joins an image's parts by itself: a launch less, for up to so many of them. Forward and backward in us,
// so / by another launch: 1 image of 300 x 192 10.0, 13.6 / 11.9, 16.3, 32 of 1000 x 48 12.7, 20.5 / 16.6, 24.3; beyond the
// bound 1 of 9216 x 96 16.6, 22.2 / 12.8, 19.5.
constexpr int kFewParts = 8192;
bool joins_itself(const GroupNormCall& a, const Deal& d)
{
    const int width = a.C / a.groups, own = d.cols * (a.dt == kBf16 ? 8 : 4);
    const int channels = d.blocks == 1 ? a.C : own + 2 * (width - 1);
    return (long)d.chunks * a.C <= kFewParts && channels <= kMostChannels;
}

// Whether the parts of a group are too many for one workgroup to join: its channels are joined over the chunks first, a launch
// more. bfloat16 images, forward and backward in us, so / by one workgroup: 1 of 1000 x 4096 in 1 group 25, 36 / 252, 476; 1 of
// 4096 x 1024 in 8 groups 24, 32 / 32, 55, in 16 23, 31 / 24, 39, in 32 (the bound) 23, 31 / 20, 32.
constexpr long kMostJoined = 16384;
bool joins_channels(const GroupNormCall& a, const Deal& d)
{
    return !joins_itself(a, d) && (long)d.chunks * (a.C / a.groups) > kMostJoined;
}
size_t joined_bytes(const GroupNormCall& a, const Deal& d)
{
    return joins_channels(a, d) ? aligned256((size_t)a.B * a.C * 16) : 0;
}
void join_channels(const GroupNormCall& a, const Deal& d, const float2* parts, const float* firsts, double2* joined,
                   hipStream_t st)
{
    hipLaunchKernelGGL(join_chunks_kernel, dim3((unsigned)((a.C + kJoinWaves - 1) / kJoinWaves), (unsigned)std::min(a.B, 32768)),
                       dim3(kJoinThreads), 0, st, a, d, parts, firsts, joined);
}

// Whether a call goes by slabs: one launch that reads a tensor once (and once more what its threads do not keep), but a
// workgroup works through its slab alone; or by passes over chunks of rows: two or three launches that read it twice. By an
// estimate in us, from the times of both at 25 shapes (1 to 64 images of 100 to 9216 rows of 48 to 1024 channels): of the 50,
// both directions, it takes the slower one by more than a tenth at four, and by less than a quarter.
bool by_slabs(const GroupNormCall& a, bool backward, const Plan& p)
{
    const Slab& s = p.s;
    if (s.cols == 0 || (long)a.B * s.slabs > (1L << 21)) return false;  // (a grid holds 2^32 threads)
    const int per = a.dt == kBf16 ? 8 : 4, most = backward ? 8 : 16;
    const bool one = s.width % per == 0;
    const double rows = std::max(1.0, (double)a.R / a.B), total = (double)a.R * a.C * (16 / per) / 5.2e6;
    // A workgroup: its latency (summing the channels of vectors in several groups takes longest), then its vectors.
    const double held = kUnits * (2048.0 / s.threads) / (p.vpt == most ? 2 : 1);  // on the chip at once
    const double rounds = std::ceil((double)a.B * s.slabs / held);
    const double vectors = rows * s.cols / s.threads, again = std::max(0.0, vectors - p.vpt);
    const double start = (backward ? (one ? 9.0 : 16.0) : (one ? 6.0 : 12.5)) * (s.threads < kSlabThreads ? 0.7 : 1.0);
    const double alone = rounds * (start + (backward ? 1.9 : 1.0) * per / 8 * (vectors + again));
    const double all = total * ((backward ? 3 : 2) + 2 * again / vectors) * 1.1;
    const double join = joins_itself(a, deal(a)) ? 0.0 : 4.0;
    const double passes = backward ? 10.5 + join + 4.5 * total : 10.5 + join + 2.6 * total;
    return std::max(alone, all) < passes;
}

// Calls go(type, activation).
template <class F>
hipError_t with_kind(const GroupNormCall& a, F&& go)
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

// ... and whether a vector lies in one group, and the vectors a thread keeps.
template <int FEW, int MANY, class F>
hipError_t with_slabs(const GroupNormCall& a, const Plan& p, F&& go)
{
    const bool one = p.s.width % (a.dt == kBf16 ? 8 : 4) == 0;
    return with_kind(a, [&](auto type, auto act) {
        constexpr std::integral_constant<int, FEW> few{};
        constexpr std::integral_constant<int, MANY> many{};
        if (one) return p.vpt == FEW ? go(type, act, std::true_type{}, few) : go(type, act, std::true_type{}, many);
        return p.vpt == FEW ? go(type, act, std::false_type{}, few) : go(type, act, std::false_type{}, many);
    });
}

hipError_t forward_by_slabs(const GroupNormCall& a, const Plan& p, const void* x, void* y, float* stats, hipStream_t st)
{
    const long items = (long)a.B * p.s.slabs;
    const dim3 grid((unsigned)((items + kXcds - 1) / kXcds * kXcds)), threads(p.s.threads);
    return with_slabs<4, 16>(a, p, [&](auto type, auto act, auto one, auto vpt) {
        hipLaunchKernelGGL((slab_kernel<decltype(type), decltype(act)::value, decltype(one)::value, decltype(vpt)::value>),
                           grid, threads, 0, st, a, p.s, static_cast<const uint8_t*>(x), static_cast<uint8_t*>(y),
                           reinterpret_cast<float2*>(stats));
        return hipGetLastError();
    });
}

hipError_t forward_by_passes(const GroupNormCall& a, const void* x, void* y, float* stats, void* ws, hipStream_t st)
{
    const Deal d = deal(a);
    char* at = static_cast<char*>(ws);
    float2* parts = reinterpret_cast<float2*>(at);
    float* firsts = reinterpret_cast<float*>(at + parts_bytes(a, d));
    float2* made = reinterpret_cast<float2*>(stats ? reinterpret_cast<char*>(stats)
                                                   : at + parts_bytes(a, d) + firsts_bytes(a));
    double2* joined = joins_channels(a, d)
                          ? reinterpret_cast<double2*>(at + parts_bytes(a, d) + firsts_bytes(a) + stats_bytes(a))
                          : nullptr;
    const bool itself = joins_itself(a, d);
    const dim3 grid((unsigned)((long)a.B * d.chunks), (unsigned)d.blocks);
    const uint8_t* xp = static_cast<const uint8_t*>(x);
    return with_kind(a, [&](auto type, auto act) {
        typedef decltype(type) S;
        hipLaunchKernelGGL((channel_moments_kernel<S>), grid, dim3(kThreads), 0, st, a, d, xp, parts, firsts);
        if (joined) join_channels(a, d, parts, firsts, joined, st);
        if (!itself)
            hipLaunchKernelGGL(group_stats_kernel, dim3(pair_groups(a)), dim3(kJoinThreads), 0, st, a, d,
                               FixedDiv((uint32_t)(a.C / a.groups)), parts, joined, firsts, made);
        hipLaunchKernelGGL((apply_kernel<S, decltype(act)::value>), grid, dim3(kThreads), 0, st, a, d, xp,
                           static_cast<uint8_t*>(y), itself ? nullptr : made, parts, firsts,
                           reinterpret_cast<float2*>(stats));
        return hipGetLastError();
    });
}

hipError_t join(const GroupNormCall& a, const float2* parts, long items, void* dw, void* db, hipStream_t st)
{
    if (!dw && !db) return hipSuccess;
    hipLaunchKernelGGL(join_sums_kernel, dim3((unsigned)((a.C + kWave - 1) / kWave)), dim3(kJoinThreads), 0, st, parts,
                       items, a.C, a.dt, dw, db);
    return hipGetLastError();
}

hipError_t backward_by_slabs(const GroupNormCall& a, const Plan& p, const void* dy, const void* x, const float* stats,
                             void* dx, void* dw, void* db, void* ws, hipStream_t st)
{
    float2* parts = static_cast<float2*>(ws);
    const long items = (long)a.B * p.s.slabs;
    const dim3 grid((unsigned)((items + kXcds - 1) / kXcds * kXcds)), threads(p.s.threads);
    const hipError_t e = with_slabs<2, 8>(a, p, [&](auto type, auto act, auto one, auto vpt) {
        hipLaunchKernelGGL(
            (slab_backward_kernel<decltype(type), decltype(act)::value, decltype(one)::value, decltype(vpt)::value>), grid,
            threads, 0, st, a, p.s, static_cast<const uint8_t*>(dy), static_cast<const uint8_t*>(x),
            static_cast<uint8_t*>(dx), reinterpret_cast<const float2*>(stats), dw || db ? parts : nullptr);
        return hipGetLastError();
    });
    return e == hipSuccess ? join(a, parts, a.B, dw, db, st) : e;
}

hipError_t backward_by_passes(const GroupNormCall& a, const void* dy, const void* x, const float* stats, void* dx, void* dw,
                              void* db, void* ws, hipStream_t st)
{
    const Deal d = deal(a);
    float2* parts = static_cast<float2*>(ws);
    float2* means = reinterpret_cast<float2*>(static_cast<char*>(ws) + parts_bytes(a, d));
    double2* joined = joins_channels(a, d)
                          ? reinterpret_cast<double2*>(static_cast<char*>(ws) + parts_bytes(a, d) + stats_bytes(a))
                          : nullptr;
    const float2* sp = reinterpret_cast<const float2*>(stats);
    const uint8_t *xp = static_cast<const uint8_t*>(x), *gp = static_cast<const uint8_t*>(dy);
    const bool itself = joins_itself(a, d);
    const dim3 grid((unsigned)((long)a.B * d.chunks), (unsigned)d.blocks);
    const hipError_t e = with_kind(a, [&](auto type, auto act) {
        typedef decltype(type) S;
        constexpr int ACT = decltype(act)::value;
        hipLaunchKernelGGL((channel_sums_kernel<S, ACT>), grid, dim3(kThreads), 0, st, a, d, gp, xp, sp, parts);
        if (joined) join_channels(a, d, parts, nullptr, joined, st);
        if (!itself)
            hipLaunchKernelGGL(group_means_kernel, dim3(pair_groups(a)), dim3(kJoinThreads), 0, st, a, d,
                               FixedDiv((uint32_t)(a.C / a.groups)), parts, joined, means);
        hipLaunchKernelGGL((input_gradient_kernel<S, ACT>), grid, dim3(kThreads), 0, st, a, d, gp, xp,
                           static_cast<uint8_t*>(dx), sp, itself ? nullptr : means, parts);
        return hipGetLastError();
    });
    return e == hipSuccess ? join(a, parts, (long)a.B * d.chunks, dw, db, st) : e;
}

}  // namespace

size_t group_norm_bytes(const GroupNormCall& a)
{
    if (by_slabs(a, false, plan(a, false))) return 0;
    const Deal d = deal(a);
    return parts_bytes(a, d) + firsts_bytes(a) + stats_bytes(a) + joined_bytes(a, d);
}

hipError_t launch_group_norm(const GroupNormCall& a, const void* x, void* y, float* stats, void* ws, hipStream_t st)
{
    const Plan p = plan(a, false);
    if (by_slabs(a, false, p)) return forward_by_slabs(a, p, x, y, stats, st);
    return forward_by_passes(a, x, y, stats, ws, st);
}

size_t group_norm_backward_bytes(const GroupNormCall& a)
{
    if (by_slabs(a, true, plan(a, true))) return aligned256((size_t)a.B * a.C * 8);
    const Deal d = deal(a);
    return parts_bytes(a, d) + stats_bytes(a) + joined_bytes(a, d);
}

hipError_t launch_group_norm_backward(const GroupNormCall& a, const void* dy, const void* x, const float* stats, void* dx,
                                      void* dw, void* db, void* ws, hipStream_t st)
{
    const Plan p = plan(a, true);
    if (by_slabs(a, true, p)) return backward_by_slabs(a, p, dy, x, stats, dx, dw, db, ws, st);
    return backward_by_passes(a, dy, x, stats, dx, dw, db, ws, st);
}

}  // namespace mpm

// Rotary positions with up to three axes: a row at grid cell (c_0, c_1, c_2) turns pair p of a head's
// channels by theta = sum_a c_a freq[a][p],
//   (o_1, o_2) = (x_1 cos - x_2 sin, x_1 sin + x_2 cos),
// and the gradients: dx is dout turned by -theta, and dfreq[a][p] the sum over rows (and heads that share
// frequencies) of c_a (x_1 dx_2 - x_2 dx_1), which needs no angle beside dx's.
// Memory bounds it: a value is read once and written once, and the angles' sines are made once for all heads of a row, in
// LDS, or by each thread where heads have frequencies of their own (one 64-bit multiply-add a pair and axis, of all three
// axes, hidden behind the loads). Queries and keys of 64 images of about 717 tokens, 12 heads of 64 each, bfloat16, in one
// launch: 53 us, 5.4 TB/s; of 8 clips of about 5700, 16 heads each with frequencies of their own, 75 us and their gradients
// 105 + 8, 5.1 and 5.5 TB/s.
#include <algorithm>
#include <type_traits>

#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {
namespace {

constexpr int kMaxThreads = 512;
constexpr int kAhead = 4;            // rows a thread loads before it turns them
constexpr int kTableBytes = 16 << 10;  // most of a workgroup's sines and cosines

// BYTES contiguous bytes as one load or store, and the float32 values in them.
template <int BYTES>
struct Piece;
template <>
struct Piece<16> {
    typedef u32x4 type;
};
template <>
struct Piece<8> {
    typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <>
struct Piece<4> {
    typedef uint32_t type;
};
template <>
struct Piece<2> {
    typedef uint16_t type;
};

// `COUNT` consecutive values of a row as they are stored.
template <class S, int COUNT>
struct Values {
    typedef typename Piece<COUNT * S::kBytes>::type Word;
    Word w;

    __device__ __forceinline__ void load(const uint8_t* p) { w = *reinterpret_cast<const Word*>(p); }
    __device__ __forceinline__ uint32_t word(int i) const
    {
        if constexpr (COUNT * S::kBytes > 4) return w[i];
        else return w;
    }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (S::kBytes == 4) return __uint_as_float(word(e));
        if constexpr (COUNT == 1) return __uint_as_float((uint32_t)w << 16);
        return e % 2 ? bf16_hi(word(e / 2)) : bf16_lo(word(e / 2));
    }
    // STREAM: past the L2.
    template <bool STREAM>
    __device__ static __forceinline__ void store(uint8_t* p, const float (&v)[COUNT])
    {
        Word w;
        if constexpr (COUNT * S::kBytes == 2) {
            w = (uint16_t)f32_to_bf16_rne(v[0]);
        } else {
            constexpr int kWords = COUNT * S::kBytes / 4;
            uint32_t u[kWords];
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (S::kBytes == 4) u[i] = __float_as_uint(v[i]);
                else u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            }
            if constexpr (kWords == 1) w = u[0];
            else
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[i] = u[i];
        }
        if constexpr (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<Word*>(p));
        else *reinterpret_cast<Word*>(p) = w;
    }
    __device__ static __forceinline__ uint32_t pack_bf16(float a, float b)
    {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 p = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
    }
};

// V pairs of a head: two runs of V values (halves), or one of 2 V (pairs).
template <class S, int V, bool HALVES>
struct Pairs {
    Values<S, HALVES ? V : 2 * V> a, b;

    __device__ __forceinline__ void load(const uint8_t* p, int pairs)
    {
        a.load(p);
        if constexpr (HALVES) b.load(p + pairs * S::kBytes);
    }
    __device__ __forceinline__ float first(int e) const { return HALVES ? a.get(e) : a.get(2 * e); }
    __device__ __forceinline__ float second(int e) const { return HALVES ? b.get(e) : a.get(2 * e + 1); }
    __device__ static __forceinline__ void store(uint8_t* p, int pairs, const float (&x)[V], const float (&y)[V])
    {
        // Neighbouring lanes write whole lines past the L2, but for halves, whose two stores it joins (8 clips of 8 x 32 x 32
        // tokens, pairs: a step 215 -> 198 us; 64 images of about 717, halves, forward 50 -> 54).
        if constexpr (HALVES) {
            Values<S, V>::template store<false>(p, x);
            Values<S, V>::template store<false>(p + pairs * S::kBytes, y);
        } else {
            float v[2 * V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[2 * e] = x[e];
                v[2 * e + 1] = y[e];
            }
            Values<S, 2 * V>::template store<true>(p, v);
        }
    }
};

// Sine and cosine of a number of turns. The turns are formed in 64 bits (a cell of thousands by a frequency
// near one leaves few digits of the fraction in 32) and only their fraction is rounded to 32. Bfloat16 values
// take the processor's sine and cosine: their error is far below the rounding of the result.
template <class S>
__device__ __forceinline__ void sine(double turns, float& sn, float& cs)
{
    const float f = (float)(turns - __builtin_rint(turns));
    if constexpr (S::kBytes == 2) {
        sn = __builtin_amdgcn_sinf(f);
        cs = __builtin_amdgcn_cosf(f);
    } else {
        sincospif(2.0f * f, &sn, &cs);
    }
}

constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)

// How the heads' pairs are dealt to the threads of a workgroup: `cols` vectors of V pairs (whole heads) side by
// side, `ways` rows at a time.
struct Deal {
    int per_head;  // vectors a head
    int cols, ways, threads;
    int blocks;      // column blocks (the grid's y)
    int tile;        // rows a workgroup turns at a time
    long tiles;
};

// The row's index in its image, and whether it belongs to one.
__device__ __forceinline__ bool image_index(const RotaryCall& a, long row, int* index)
{
    if (!a.off) {
        *index = (int)(row % a.N);
        return true;
    }
    if (row < a.off[0] || row >= a.off[a.B]) return false;
    int lo = 0, hi = a.B;  // off[lo] <= row < off[hi]
    if (!a.pos) {
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.off[mid] <= row) lo = mid;
            else hi = mid;
        }
    }
    *index = (int)(row - a.off[lo]);
    return true;
}

// A workgroup's rows and heads.
struct RowsAt {
    long first;
    int rows, head, heads;
};

// `many` bytes from `from` on of each head as they are (zeros in rows that are not turned, if they are written): a thread
// has one piece of BYTES of a head and walks the rows. 40000 rows of 4 heads of 80 channels, 32 of them turned, 17.5 us (one word
// of four bytes after another of all rows 31.7); 45875 of 24 of 64, half of them 81 (113).
template <class S, int BYTES>
__device__ __forceinline__ void pass_channels(const RotaryCall& a, const HeadRows& src, const HeadRows& dst, const RowsAt& at,
                                              int from, int many, bool zero, const int* cells)
{
    typedef typename Piece<BYTES>::type Word;
    const int words = many / BYTES, cols = min(at.heads, a.H - at.head) * words, threads = blockDim.x, t = threadIdx.x;
    const int step = max(1, threads / cols), first = step > 1 ? t / cols : 0;  // rows at a time, and this thread's first
    if (first >= step) return;
    for (int c = t - first * cols; c < cols; c += step > 1 ? cols : threads) {
        const int h = c / words;
        const long in = from + (long)(c - h * words) * BYTES, head = at.head + h;
        const uint8_t* p = src.p + (at.first * src.row + head * src.head) * S::kBytes + in;
        uint8_t* q = dst.p + (at.first * dst.row + head * dst.head) * S::kBytes + in;
        for (int r = first; r < at.rows; r += kAhead * step) {
            Word w[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                w[u] = *reinterpret_cast<const Word*>(p + (long)min(r + u * step, at.rows - 1) * src.row * S::kBytes);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int row = r + u * step;
                if (row >= at.rows) break;
                const bool turned = cells[4 * row + 3];
                if (turned || zero) *reinterpret_cast<Word*>(q + (long)row * dst.row * S::kBytes) = turned ? w[u] : Word{};
            }
        }
    }
}

// GRAD: src is dout and x the forward call's rows; the workgroup's sums of c_a (x_1 dx_2 - x_2 dx_1) go to
// parts[workgroup][head or 1][axis][pair]. `sign` turns the other way, `zero` writes zeros to rows of no image.
template <class S, int V, bool HALVES, bool PER_HEAD, bool GRAD>
__global__ __launch_bounds__(kMaxThreads) void rotary_kernel(RotaryCall a, HeadRows src, HeadRows x, HeadRows dst,
                                                             float sign, bool zero, Deal d, float* __restrict__ parts)
{
    typedef Pairs<S, V, HALVES> P;
    extern __shared__ __align__(16) uint8_t lds[];
    int* cells = reinterpret_cast<int*>(lds);                          // [tile][4]: three coordinates, whether it is turned
    float2* table = reinterpret_cast<float2*>(lds + d.tile * 16);      // [tile][pairs]: sine, cosine
    const int t = threadIdx.x, way = t / d.cols, local = t - way * d.cols, j = local % d.per_head;
    const int head = blockIdx.y * (d.cols / d.per_head) + local / d.per_head;
    const bool active = way < d.ways && head < a.H;
    const long at = (long)head * S::kBytes, in_head = (long)j * V * (HALVES ? 1 : 2) * S::kBytes;

    double freq[PER_HEAD ? kMaxAxes : 1][PER_HEAD ? V : 1];
    if constexpr (PER_HEAD) {
#pragma unroll
        for (int i = 0; i < kMaxAxes; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e)
                freq[i][e] = active && i < a.axes
                                 ? kTurn * (double)a.freq[((long)head * a.axes + i) * a.pairs + j * V + e]
                                 : 0.0;
    }
    float sums[GRAD ? kMaxAxes : 1][GRAD ? V : 1];
    if constexpr (GRAD) {
#pragma unroll
        for (int i = 0; i < kMaxAxes; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[i][e] = 0.0f;
    }

    for (long tile = blockIdx.x; tile < d.tiles; tile += gridDim.x) {
        const long r0 = tile * d.tile;
        const int rows = (int)min((long)d.tile, (long)a.R - r0);
        __syncthreads();  // the tile before has been read
        for (int r = t; r < rows; r += blockDim.x) {
            int index = 0, c[kMaxAxes] = {0, 0, 0};
            const bool turned = image_index(a, r0 + r, &index);
            if (turned && a.pos) index = a.pos[r0 + r];
            long limit = 1;
            for (int i = 0; i < a.axes; ++i) limit *= a.grid[i];
            index = (int)min(max((long)index, 0L), limit - 1);
#pragma unroll
            for (int i = kMaxAxes - 1; i > 0; --i) {
                if (i < a.axes) {
                    c[i] = index % a.grid[i];
                    index /= a.grid[i];
                }
            }
            c[0] = index;
            *reinterpret_cast<int4*>(cells + 4 * r) = make_int4(c[0], c[1], c[2], turned);
        }
        __syncthreads();
        if constexpr (!PER_HEAD) {
            for (int e = t; e < rows * a.pairs; e += blockDim.x) {
                const int r = e / a.pairs, p = e - r * a.pairs;
                double turns = 0.0;
                for (int i = 0; i < a.axes; ++i)
                    turns = fma((double)cells[4 * r + i], (double)a.freq[i * a.pairs + p], turns);
                float sn, cs;
                sine<S>(turns * kTurn, sn, cs);
                table[e] = make_float2(sn, cs);
            }
            __syncthreads();
        }
        if (active) {
            for (int base = way; base < rows; base += d.ways * kAhead) {
                P in[kAhead], xs[GRAD ? kAhead : 1];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const long row = r0 + min(base + u * d.ways, rows - 1);
                    in[u].load(src.p + row * src.row * S::kBytes + at * src.head + in_head, a.pairs);
                    if constexpr (GRAD) xs[u].load(x.p + row * x.row * S::kBytes + at * x.head + in_head, a.pairs);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int r = base + u * d.ways;
                    if (r >= rows) break;
                    const int4 cell = *reinterpret_cast<const int4*>(cells + 4 * r);
                    if (!cell.w && !zero) continue;
                    float o1[V], o2[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float sn, cs;
                        if constexpr (PER_HEAD) {
                            const double turns = fma((double)cell.x, freq[0][e],
                                                     fma((double)cell.y, freq[1][e], (double)cell.z * freq[2][e]));
                            sine<S>(turns, sn, cs);
                        } else {
                            const float2 sc = table[r * a.pairs + j * V + e];
                            sn = sc.x;
                            cs = sc.y;
                        }
                        sn *= sign;
                        const float p = in[u].first(e), q = in[u].second(e);
                        o1[e] = cell.w ? fmaf(p, cs, -q * sn) : 0.0f;
                        o2[e] = cell.w ? fmaf(p, sn, q * cs) : 0.0f;
                        if constexpr (GRAD) {
                            const float g = cell.w ? fmaf(xs[u].first(e), o2[e], -xs[u].second(e) * o1[e]) : 0.0f;
                            sums[0][e] = fmaf((float)cell.x, g, sums[0][e]);
                            sums[1][e] = fmaf((float)cell.y, g, sums[1][e]);
                            sums[2][e] = fmaf((float)cell.z, g, sums[2][e]);
                        }
                    }
                    const long row = r0 + r;
                    P::store(dst.p + row * dst.row * S::kBytes + at * dst.head + in_head, a.pairs, o1, o2);
                }
            }
        }
        // The channels that pass, in the widest pieces that their start and number allow (two channels a pair: four bytes).
        const int from = 2 * a.pairs * S::kBytes, many = a.dh * S::kBytes - from;
        if (many > 0 && (zero || src.p != dst.p)) {
            const RowsAt at{r0, rows, (int)blockIdx.y * (d.cols / d.per_head), d.cols / d.per_head};
            if ((from | many) % 16 == 0) pass_channels<S, 16>(a, src, dst, at, from, many, zero, cells);
            else if ((from | many) % 8 == 0) pass_channels<S, 8>(a, src, dst, at, from, many, zero, cells);
            else pass_channels<S, 4>(a, src, dst, at, from, many, zero, cells);
        }
    }

    if constexpr (GRAD) {
        // The sums of threads with the same pairs (and head), in order, by way of LDS: [axis][e][thread].
        float* all = reinterpret_cast<float*>(lds);
        const int threads = blockDim.x;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMaxAxes; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (i < a.axes) all[(i * V + e) * threads + t] = active ? sums[i][e] : 0.0f;
        __syncthreads();
        const int heads = d.cols / d.per_head, h0 = blockIdx.y * heads;
        const int keep = PER_HEAD ? min(heads, a.H - h0) : 1;         // heads that have sums of their own
        const int step = PER_HEAD ? d.cols : d.per_head, many = PER_HEAD ? d.ways : d.ways * heads;
        const long group = PER_HEAD ? (long)blockIdx.x * a.H + h0 : (long)blockIdx.x * d.blocks + blockIdx.y;
        for (int o = t; o < keep * a.axes * a.pairs; o += threads) {
            const int h = o / (a.axes * a.pairs), i = o / a.pairs % a.axes, p = o % a.pairs;
            const float* from = all + (i * V + p % V) * threads + h * d.per_head + p / V;
            float s = 0.0f;
            for (int k = 0; k < many; ++k) s += from[k * step];
            parts[group * a.axes * a.pairs + o] = s;
        }
    }
}

// dfreq: the workgroups' parts summed in order, 16 threads a value, in 64 bits.
__global__ __launch_bounds__(1024) void join_frequencies_kernel(const float* __restrict__ parts, long groups, int values,
                                                                float* __restrict__ out)
{
    constexpr int kCols = 64, kWays = 16;
    __shared__ double lds[kWays][kCols];
    const int lane = threadIdx.x % kCols, way = threadIdx.x / kCols, col = blockIdx.x * kCols + lane;
    double s = 0.0;
    if (col < values) {
#pragma unroll 4
        for (long g = way; g < groups; g += kWays) s += (double)parts[g * values + col];
    }
    lds[way][lane] = s;
    __syncthreads();
    if (way != 0 || col >= values) return;
    for (int w = 1; w < kWays; ++w) s += lds[w][lane];
    out[col] = (float)s;
}

// Workgroups of a backward pass with frequencies' gradients, and of bfloat16 calls with frequencies by head, which a thread
// then reads once for many rows: us so / with a workgroup a tile 45875 rows of 32 heads of 64 73 / 83 (512 workgroups 93),
// of 24 59 / 71, 100000 of 8 of 128 86 / 118, 60000 of 4 of 32 10.8 / 10.8; float32, whose sines take longest, 57 / 52.
constexpr int kGradGroups = 1024;

// V pairs a vector.
Deal deal(const RotaryCall& a, int V)
{
    Deal d;
    d.per_head = a.pairs / V;
    const int whole = a.H * d.per_head;
    if (whole <= kMaxThreads) {
        // As many rows at a time as leave the fewest lanes idle, in 192 threads or more where rows allow.
        d.cols = whole;
        d.ways = 1;
        double best = 0.0;
        for (int w = 1; w * whole <= kMaxThreads; ++w) {
            const int threads = (w * whole + kWave - 1) / kWave * kWave;
            double use = (double)(w * whole) / threads;
            if (threads < 192) use *= threads / 192.0;
            if (use > best + 0.01) {
                best = use;
                d.ways = w;
            }
        }
    } else {
        d.cols = std::max(1, 256 / d.per_head) * d.per_head;
        d.ways = 1;
    }
    d.threads = (d.ways * d.cols + kWave - 1) / kWave * kWave;
    d.blocks = (whole + d.cols - 1) / d.cols;
    // Rows a tile: kAhead of a thread's, within the table's bytes, and few enough for two workgroups a compute unit.
    long rows = d.ways * kAhead;
    if (!a.per_head) rows = std::min(rows, std::max(1L, (long)kTableBytes / (8L * a.pairs)));
    rows = std::min(rows, std::max((long)d.ways, ((long)a.R * d.blocks + 511) / 512));
    d.tile = (int)std::max(1L, rows);
    d.tiles = ((long)a.R + d.tile - 1) / d.tile;
    return d;
}

long grad_groups(const Deal& d) { return std::min(d.tiles, std::max(1L, (long)kGradGroups / d.blocks)); }

// The pairs a vector: the widest that divides a head's.
int vector_pairs(const RotaryCall& a)
{
    int v = a.dt == kBf16 ? 8 : 4;
    if (!a.halves) v /= 2;
    while (a.pairs % v != 0) v /= 2;
    return v;
}

template <class S, int V, bool HALVES, bool PER_HEAD, bool GRAD>
hipError_t launch_one(const RotaryCall& a, const HeadRows& src, const HeadRows& x, const HeadRows& dst, bool inverse,
                      bool zero, float* parts, hipStream_t st)
{
    const Deal d = deal(a, V);
    size_t bytes = (size_t)d.tile * 16 + (PER_HEAD ? 0 : (size_t)d.tile * a.pairs * 8);
    if (GRAD) bytes = std::max(bytes, (size_t)a.axes * V * d.threads * 4);
    const bool keeps = GRAD || (PER_HEAD && S::kBytes == 2);
    const long groups = keeps ? grad_groups(d) : std::min(d.tiles, 1L << 22);  // (a grid holds 2^32 threads)
    hipLaunchKernelGGL((rotary_kernel<S, V, HALVES, PER_HEAD, GRAD>), dim3((unsigned)groups, (unsigned)d.blocks),
                       dim3(d.threads), bytes, st, a, src, x, dst, inverse ? -1.0f : 1.0f, zero, d, parts);
    return hipGetLastError();
}

template <class S, int V, bool HALVES>
hipError_t launch_layout(const RotaryCall& a, const HeadRows& src, const HeadRows& x, const HeadRows& dst, bool inverse,
                         bool zero, float* parts, hipStream_t st)
{
    if (parts)
        return a.per_head ? launch_one<S, V, HALVES, true, true>(a, src, x, dst, inverse, zero, parts, st)
                          : launch_one<S, V, HALVES, false, true>(a, src, x, dst, inverse, zero, parts, st);
    return a.per_head ? launch_one<S, V, HALVES, true, false>(a, src, x, dst, inverse, zero, parts, st)
                      : launch_one<S, V, HALVES, false, false>(a, src, x, dst, inverse, zero, parts, st);
}

hipError_t launch_any(const RotaryCall& a, const HeadRows& src, const HeadRows& x, const HeadRows& dst, bool inverse,
                      bool zero, float* parts, hipStream_t st)
{
    const int v = vector_pairs(a);
#define MPM_ROTARY(S, V, HALVES) return launch_layout<S, V, HALVES>(a, src, x, dst, inverse, zero, parts, st)
    if (a.dt == kBf16) {
        if (a.halves) {
            if (v == 8) MPM_ROTARY(Bf16, 8, true);
            if (v == 4) MPM_ROTARY(Bf16, 4, true);
            if (v == 2) MPM_ROTARY(Bf16, 2, true);
            MPM_ROTARY(Bf16, 1, true);
        }
        if (v == 4) MPM_ROTARY(Bf16, 4, false);
        if (v == 2) MPM_ROTARY(Bf16, 2, false);
        MPM_ROTARY(Bf16, 1, false);
    }
    if (a.halves) {
        if (v == 4) MPM_ROTARY(F32, 4, true);
        if (v == 2) MPM_ROTARY(F32, 2, true);
        MPM_ROTARY(F32, 1, true);
    }
    if (v == 2) MPM_ROTARY(F32, 2, false);
    MPM_ROTARY(F32, 1, false);
#undef MPM_ROTARY
}

}  // namespace

hipError_t launch_rotary(const RotaryCall& a, const HeadRows& x, const HeadRows& out, bool inverse, hipStream_t stream)
{
    return launch_any(a, x, HeadRows{nullptr, 0, 0}, out, inverse, false, nullptr, stream);
}

size_t rotary_backward_bytes(const RotaryCall& a)
{
    const Deal d = deal(a, vector_pairs(a));
    return (size_t)grad_groups(d) * (a.per_head ? a.H : d.blocks) * a.axes * a.pairs * 4;
}

hipError_t launch_rotary_backward(const RotaryCall& a, const HeadRows& dout, const HeadRows& x, const HeadRows& dx,
                                  float* dfreq, void* ws, hipStream_t stream)
{
    float* parts = dfreq ? static_cast<float*>(ws) : nullptr;
    hipError_t e = launch_any(a, dout, x, dx, true, true, parts, stream);
    if (e != hipSuccess || !dfreq) return e;
    const Deal d = deal(a, vector_pairs(a));
    const int values = (a.per_head ? a.H : 1) * a.axes * a.pairs;
    hipLaunchKernelGGL(join_frequencies_kernel, dim3((unsigned)((values + 63) / 64)), dim3(1024), 0, stream, parts,
                       grad_groups(d) * (a.per_head ? 1 : d.blocks), values, dfreq);
    return hipGetLastError();
}

}  // namespace mpm

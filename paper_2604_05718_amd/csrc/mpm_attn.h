// Shared by the attention kernels: the call's layout, tiles in LDS, matrix fragments.
//
// Matrix products run on 32 x 32 MFMA tiles. A wave holds its 32 own rows (queries in the
// forward and query-gradient kernels, keys in the key-gradient kernel) as the B operand, so
// that in every score tile a lane owns one of them (lane % 32) and 16 rows of the other side:
// register r of half h = lane / 32 is row 8 (r / 4) + 4 h + r % 4. A score tile is then the B
// operand of the next product without leaving its registers: a step of 16 contracted rows
// takes registers 8 s ... 8 s + 7, rows 16 s + 8 (i / 4) + 4 h + i % 4 of element i, and the A
// operand's rows are read in that order (cols_frag).
#pragma once

#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Eight consecutive values along the contracted axis of a 32 x 32 x 16 product step, for one
// lane: rows of one operand lane % 32, contracted indices 8 (lane / 32) ... + 7.
template <class S> struct FragOf;
template <> struct FragOf<Bf16> { typedef bf16x8 type; };
template <> struct FragOf<F32> { typedef f32x8 type; };

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Float32: eight products of contracted depth 2, element i of both halves in one.
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// A tile of rows of DH values in LDS. Rows hold 16-byte chunks; chunk c of row r is stored at
// chunk c ^ mix(r), so that the 16 rows one phase of a wave's 16-byte reads covers hit all 64
// banks once, and the 8 rows x 64 bytes of a transposing read hit each bank twice (its least).
template <class S, int DH>
struct Tile {
    static constexpr int kRowBytes = DH * S::kBytes;
    static constexpr int kChunks = kRowBytes / 16;

    __device__ static __forceinline__ int mix(int r)
    {
        if constexpr (kChunks == 4) return ((r >> 2) & 1) * 2 + ((r >> 3) & 1);
        if constexpr (kChunks == 8) return ((r >> 1) & 1) * 4 + ((r >> 2) & 1) * 2 + ((r >> 3) & 1);
        return (r & 1) * 8 + ((r >> 1) & 1) * 4 + ((r >> 2) & 1) * 2 + ((r >> 3) & 1);
    }
    __device__ static __forceinline__ int at(int r, int c) { return r * kRowBytes + ((c ^ mix(r)) << 4); }
};


// Contracted step s of row r (lane % 32 of its 32-row group): values 16 s + 8 h ... + 7 of it.
template <class S, int DH>
__device__ __forceinline__ typename FragOf<S>::type rows_frag(const uint8_t* tile, int r, int s, int h)
{
    typedef Tile<S, DH> T;
    if constexpr (S::kBytes == 2) {
        return __builtin_bit_cast(bf16x8, load16(tile + T::at(r, 2 * s + h)));
    } else {
        const f32x4 a = __builtin_bit_cast(f32x4, load16(tile + T::at(r, 4 * s + 2 * h)));
        const f32x4 b = __builtin_bit_cast(f32x4, load16(tile + T::at(r, 4 * s + 2 * h + 1)));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// The transposed operand: column d0 + lane % 32 of rows r0 + 8 (i / 4) + 4 h + i % 4, i < 8 (r0 a
// multiple of 16). Bfloat16: two transposing reads, each giving a group of 16 lanes one column
// each of a 4 x 16 block whose rows the group's lanes address, four lanes a row.
template <class S, int DH>
__device__ __forceinline__ typename FragOf<S>::type cols_frag(const uint8_t* tile, int r0, int d0, int lane)
{
    typedef Tile<S, DH> T;
    const int h = lane >> 5;
    if constexpr (S::kBytes == 2) {
        const int d = d0 + (lane & 16) + 4 * (lane & 3);
        const int r = r0 + 4 * h + ((lane & 15) >> 2);
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        s16x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            v[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s16x4*)(tile + T::at(r + 8 * u, d >> 3) + (d & 7) * 2));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 w = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(bf16x8, w);
    } else {
        const int d = d0 + (lane & 31);
        f32x8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = *reinterpret_cast<const float*>(tile + T::at(r0 + 8 * (i >> 2) + 4 * h + (i & 3), d >> 2) + (d & 3) * 4);
        return w;
    }
}

// Registers 8 s ... 8 s + 7 of a score tile as an operand; bfloat16: rounded to nearest even, as the matrix
// instruction takes both operands in one type. With the output's own rounding a forward result is off by 0.0023 of
// its norm, against 0.0017 for unrounded probabilities; a second product for what is rounded off would be half as
// many again.
__device__ __forceinline__ bf16x8 tile_frag(const f32x16& p, int s, Bf16)
{
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const f32x2 v = {p[8 * s + i], p[8 * s + i + 1]};
        const bf16x2 b = __builtin_convertvector(v, bf16x2);
        w[i] = b[0];
        w[i + 1] = b[1];
    }
    return w;
}
__device__ __forceinline__ f32x8 tile_frag(const f32x16& p, int s, F32)
{
    f32x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = p[8 * s + i];
    return w;
}

// Adds the eight values of such an operand. A row's probabilities are divided by the sum of what was multiplied: with
// the sum of the unrounded ones a row that one key has all of would come out as that key's values times a rounding.
__device__ __forceinline__ float frag_sum(bf16x8 p, float sum)
{
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const bf16x2 v = {p[i], p[i + 1]};
        sum = __builtin_amdgcn_fdot2_f32_bf16(v, one, sum, false);
    }
    return sum;
}
__device__ __forceinline__ float frag_sum(f32x8, float sum) { return sum; }

// Sum and maximum of a value over the two halves of a wave (lanes l and l ^ 32).
__device__ __forceinline__ float halves_max(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float halves_sum(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// One 16-byte chunk of a row of dh values: zero past the row's end or for a row that is not live.
template <class S>
__device__ __forceinline__ u32x4 load_chunk(const uint8_t* row, int c, int dh, bool live)
{
    u32x4 v = {0, 0, 0, 0};
    if (live && c * (16 / S::kBytes) < dh) v = load16(row + c * 16);
    return v;
}

// The rows of one operand fragment set straight from memory: row r's values 16 s + 8 h ... for all s.
template <class S, int DH>
__device__ __forceinline__ void load_frags(typename FragOf<S>::type (&f)[DH / 16], const uint8_t* row, int dh,
                                           bool live, int h)
{
#pragma unroll
    for (int s = 0; s < DH / 16; ++s) {
        if constexpr (S::kBytes == 2) {
            f[s] = __builtin_bit_cast(bf16x8, load_chunk<S>(row, 2 * s + h, dh, live));
        } else {
            const f32x4 a = __builtin_bit_cast(f32x4, load_chunk<S>(row, 4 * s + 2 * h, dh, live));
            const f32x4 b = __builtin_bit_cast(f32x4, load_chunk<S>(row, 4 * s + 2 * h + 1, dh, live));
            f[s] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
}

// Stores a wave's 32 result rows from product tiles: lane's row (lane % 32) at `row`, column
// 32 d + 8 g + 4 h + e of it in register 4 g + e of tile d, times f, rounded to nearest even.
// Bfloat16: the halves of a wave exchange their four-column pieces of two groups, so that every
// store is 16 bytes of one row.
template <int D>
__device__ __forceinline__ void store_rows(uint8_t* row, const f32x16 (&x)[D], float f, int dh, bool live, int h, Bf16)
{
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const f32x2 a = {x[d][4 * g + 2 * j] * f, x[d][4 * g + 2 * j + 1] * f};
                const f32x2 b = {x[d][4 * g + 4 + 2 * j] * f, x[d][4 * g + 5 + 2 * j] * f};
                const auto p = __builtin_amdgcn_permlane32_swap(
                    __builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2)),
                    __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2)), false, false);
                w[j] = p[0];
                w[2 + j] = p[1];
            }
            const int at = 32 * d + 8 * (g + h);
            if (live && at < dh) store16(row + at * 2, w);
        }
}
template <int D>
__device__ __forceinline__ void store_rows(uint8_t* row, const f32x16 (&x)[D], float f, int dh, bool live, int h, F32)
{
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = 32 * d + 8 * g + 4 * h;
            if (live && at < dh)
                *reinterpret_cast<float4*>(row + at * 4) =
                    make_float4(x[d][4 * g] * f, x[d][4 * g + 1] * f, x[d][4 * g + 2] * f, x[d][4 * g + 3] * f);
        }
}

// Row range of image b (the same in all lanes of a wave): packed offsets or N rows each, its count held to [0, N].
struct Rows {
    long first;
    int count;
};
__device__ __forceinline__ Rows image_rows(const int32_t* off, int b, int N)
{
    if (off == nullptr) return Rows{(long)b * N, N};
    // (the same for every lane: kept in scalar registers)
    const int o = __builtin_amdgcn_readfirstlane(off[b]), e = __builtin_amdgcn_readfirstlane(off[b + 1]);
    return Rows{(long)o, min(max(e - o, 0), N)};
}
// ... of images that differ between lanes.
__device__ __forceinline__ Rows lane_rows(const int32_t* off, int b, int N)
{
    if (off == nullptr) return Rows{(long)b * N, N};
    const int o = off[b];
    return Rows{(long)o, min(max(off[b + 1] - o, 0), N)};
}

// How a kernel takes the position bias of a pair.
enum BiasKind : int {
    kBiasNone = 0,
    kBiasGrid = 1,  // no offset of the grid is past the span: one subtraction an entry
    kBiasFar = 2    // offsets are held to the span, one axis at a time
};

// A grid position in the form its side of the bias entry needs (entries of 4 bytes).
// kBiasGrid: the byte offset of row * W + column (W = 2 span + 1), so that a pair's entry is
// query - key + middle. kBiasFar:
// row and column as two 16-bit halves. Positions outside the grid are held to it, so that a
// pair's entry is inside the table whatever the caller passed.
template <int BIAS>
__device__ __forceinline__ int bias_code(int pos, int gh, int gw, int W)
{
    if constexpr (BIAS == kBiasNone) return 0;
    const int p = min(max(pos, 0), gh * gw - 1);
    const int r = (int)((unsigned)p / (unsigned)gw), c = p - r * gw;
    if constexpr (BIAS == kBiasGrid) return (r * W + c) * 4;
    return (r << 16) | c;
}
// Where the pair's entry is: qcode's side holds the table's address (kBiasFar: base does).
template <int BIAS>
__device__ __forceinline__ int bias_entry(int qcode, int kcode, int span, int W, int base)
{
    if constexpr (BIAS == kBiasGrid) return qcode - kcode;
    const int dr = (qcode >> 16) - (kcode >> 16), dc = (qcode & 0xffff) - (kcode & 0xffff);
    return base + ((min(max(dr, -span), span) + span) * W + min(max(dc, -span), span) + span) * 4;
}
// A query's side: with the middle of the table at LDS address `base` added (kBiasGrid).
template <int BIAS>
__device__ __forceinline__ int query_code(int pos, int gh, int gw, int span, int W, int base)
{
    const int c = bias_code<BIAS>(pos, gh, gw, W);
    return BIAS == kBiasGrid ? c + (span * W + span) * 4 + base : c;
}

// An LDS address as the 32-bit number the hardware takes, and a float at one: a pair's bias is read at
// the table's address plus its entry, whose query part holds the address already.
typedef __attribute__((address_space(3))) const float lds_float;
__device__ __forceinline__ int lds_address(const void* p)
{
    return (int)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p;
}
__device__ __forceinline__ float lds_at(int address) { return *(lds_float*)(uintptr_t)(uint32_t)address; }

// A score term in the exponent's base: x log2(e), a finite value kept finite (a mask may use the
// type's lowest value, whose rows then average all of their keys as the softmax of equal scores, or its
// highest): beyond 2.35e38 in magnitude it counts as that.
__device__ __forceinline__ float to_log2(float x)
{
    const float y = x * kLog2e;
    return fabsf(x) <= -kLowest ? __builtin_amdgcn_fmed3f(y, kLowest, -kLowest) : y;
}

constexpr int kXcds = 8;
// The workgroup's row block and (image, head) pair. Blocks are dealt round-robin to the 8 XCDs,
// each with its own L2: pairs are dealt to XCDs whole, so that the blocks that read one pair's
// rows share an L2 (few pairs: in order, since whole pairs would leave XCDs idle).
__device__ __forceinline__ bool block_item(int blocks, long pairs, int* blk, int* pair)
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
// Workgroups of such a launch.
inline long block_grid(long pairs, int blocks)
{
    return (pairs >= 4 * kXcds ? (pairs + kXcds - 1) / kXcds * kXcds : pairs) * blocks;
}

// Tiles of ROWS rows of two operands on their way to LDS: loaded to registers a tile ahead. SCALAR: a whole
// tile's loads take a scalar address and an offset of the thread's own, the same for every tile; otherwise
// each thread walks its chunks by their addresses (the key kernel, whose scalar registers are full: 640
// against 690 us on 3 images of 4096 tokens, where the other two kernels gain 2 to 4%).
template <class S, int DH, int ROWS, int THREADS, bool SCALAR>
struct PairStage {
    typedef Tile<S, DH> T;
    static constexpr int kTileBytes = ROWS * T::kRowBytes;
    static constexpr int kPer = ROWS * T::kChunks / THREADS;
    static_assert(ROWS * T::kChunks % THREADS == 0 && THREADS >= ROWS, "whole chunks a thread");
    u32x4 x[kPer], y[kPer];
    float dropped[kPer];
    const uint8_t *xb, *yb;  // the first row
    long xs, ys;             // bytes from row to row
    uint32_t xo[kPer], yo[kPer];
    bool narrow;  // offsets inside a tile fit 32 bits, rows are whole
    const uint8_t *xp[kPer], *yp[kPer];  // (not SCALAR) the chunks of the next tile

    __device__ __forceinline__ void init(const HeadRows& xr, const HeadRows& yr, long first, int head, int dh, int t)
    {
        xs = xr.row * S::kBytes;
        ys = yr.row * S::kBytes;
        xb = xr.p + first * xs + (long)head * xr.head * S::kBytes;
        yb = yr.p + first * ys + (long)head * yr.head * S::kBytes;
        constexpr long kMost = (1L << 31) / ROWS;
        narrow = dh == DH && xs < kMost && ys < kMost;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = t + i * THREADS;
            xo[i] = (uint32_t)(e / T::kChunks) * (uint32_t)xs + e % T::kChunks * 16;
            yo[i] = (uint32_t)(e / T::kChunks) * (uint32_t)ys + e % T::kChunks * 16;
            if (!SCALAR) {
                xp[i] = xb + e / T::kChunks * xs + e % T::kChunks * 16;
                yp[i] = yb + e / T::kChunks * ys + e % T::kChunks * 16;
            }
        }
    }
    // Loads rows r0 ... of `count` (tiles in order); zeros past the last row and past a row's end. Rows dropped by
    // drop[row] = -inf are stored as zeros, whatever they hold (loaded all the same: a load that
    // waits for its drop value would take twice the latency).
    template <bool DROP>
    __device__ __forceinline__ void load(int dh, int count, const float* drop, int r0, int t)
    {
        const uint8_t *xt = xb + r0 * xs, *yt = yb + r0 * ys;
        if (SCALAR && narrow && r0 + ROWS <= count) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                x[i] = load16(xt + xo[i]);
                y[i] = load16(yt + yo[i]);
                if (DROP) dropped[i] = drop[r0 + (t + i * THREADS) / T::kChunks];
            }
            return;
        }
        const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = t + i * THREADS, ch = e % T::kChunks, r = e / T::kChunks;
            x[i] = y[i] = zero;
            if (DROP) dropped[i] = 0.0f;
            if (ch * (16 / S::kBytes) < dh && r0 + r < count) {
                if (DROP) dropped[i] = drop[r0 + r];
                x[i] = load16(SCALAR ? xt + r * xs + ch * 16 : xp[i]);
                y[i] = load16(SCALAR ? yt + r * ys + ch * 16 : yp[i]);
            }
            if (!SCALAR) {
                xp[i] += ROWS * xs;
                yp[i] += ROWS * ys;
            }
        }
    }
    template <bool DROP>
    __device__ __forceinline__ void store(uint8_t* lds, int t)
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (DROP && dropped[i] == -__builtin_inff()) {
                const u32x4 zero = {0, 0, 0, 0};
                x[i] = y[i] = zero;
            }
            const int e = t + i * THREADS, at = T::at(e / T::kChunks, e % T::kChunks);
            store16(lds + at, x[i]);
            store16(lds + kTileBytes + at, y[i]);
        }
    }
};

// A head's bias table to LDS, in base 2: sixteen loads a thread in flight.
template <int THREADS>
__device__ __forceinline__ void load_table(float* table, const float* src, int n, int t)
{
    constexpr int kFlight = 16;
    for (int e0 = t; e0 < n; e0 += THREADS * kFlight) {
        float v[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) v[i] = src[min(e0 + i * THREADS, n - 1)];
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (e0 + i * THREADS < n) table[e0 + i * THREADS] = to_log2(v[i]);
    }
}

}  // namespace mpm

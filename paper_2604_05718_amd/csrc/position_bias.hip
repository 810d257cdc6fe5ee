// The learned relative position bias by buckets: a table of nb x nb entries a head, indexed by
// the buckets of a row and a column offset, laid out by offset for the attention kernels, and
// the gradient back from that layout to the table.
#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float table_value(const void* p, long i, int dt)
{
    if (dt == kBf16) return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
    return reinterpret_cast<const float*>(p)[i];
}

// bias[h][r][c] = table[lut[r] nb + lut[c]][h]: one thread an entry, entries along the row of
// one head, so that stores are whole lines (the table, at most a few hundred KB, is read from L2).
// A launch of 3 to 6 us, bound by its latency: 16 heads of 127 x 127 offsets are 1 MB.
__global__ __launch_bounds__(kThreads) void bias_expand_kernel(const void* __restrict__ table,
                                                               const int32_t* __restrict__ lut, int nb, int W, int H,
                                                               int dt, float* __restrict__ bias)
{
    const int e = blockIdx.x * kThreads + threadIdx.x;
    if (e >= W * W) return;
    const int h = blockIdx.y;
    const int r = min(max(lut[e / W], 0), nb - 1), c = min(max(lut[e % W], 0), nb - 1);
    bias[(long)h * W * W + e] = table_value(table, ((long)r * nb + c) * H + h, dt);
}

// dtable[bucket][h] = sum of dbias[h] over the bucket's offsets: a workgroup takes a row bucket of
// a head. The row offsets that have it are listed; every thread adds its column offset's entries of
// those rows, in order; then a thread a column bucket adds its columns' sums, in order. 16 heads of
// 127 x 127 offsets 13 us, 12 of 63 x 63 8 us, each a chain of loads and adds of one row bucket.
constexpr int kMaxWidth = 128;
__global__ __launch_bounds__(kMaxWidth) void bias_gradient_kernel(const float* __restrict__ dbias,
                                                                  const int32_t* __restrict__ lut, int nb, int W, int H,
                                                                  int dt, void* __restrict__ dtable)
{
    constexpr int kFlight = 8;
    __shared__ int32_t axis[kMaxWidth];
    __shared__ float sums[kMaxWidth];
    __shared__ int32_t rows[kMaxWidth];
    __shared__ int32_t first_wave;
    const int t = threadIdx.x, lane = t % kWave, br = blockIdx.x, h = blockIdx.y;
    const int32_t own = t < W ? lut[t] : -1;
    axis[t] = own;
    const unsigned long long has = __ballot(own == br);
    const int before = __popcll(has & ((1ull << lane) - 1));
    if (t == 0) first_wave = __popcll(has);
    __syncthreads();
    if (own == br) rows[before + (t >= kWave ? first_wave : 0)] = t;
    const int count = __syncthreads_count(own == br);
    float sum = 0.0f;
    const float* col = dbias + (long)h * W * W + min(t, W - 1);
    for (int i = 0; i < count; i += kFlight) {
        float v[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) v[u] = col[(long)rows[min(i + u, count - 1)] * W];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (i + u < count) sum += v[u];
    }
    sums[t] = sum;
    __syncthreads();
    if (t >= nb) return;
    sum = 0.0f;
    for (int c = 0; c < W; ++c)
        if (axis[c] == t) sum += sums[c];
    const long at = ((long)br * nb + t) * H + h;
    if (dt == kBf16) reinterpret_cast<uint16_t*>(dtable)[at] = (uint16_t)f32_to_bf16_rne(sum);
    else reinterpret_cast<float*>(dtable)[at] = sum;
}

}  // namespace

hipError_t launch_bias_expand(const void* table, const int32_t* lut, int nb, int span, int H, int dt, float* bias,
                              hipStream_t stream)
{
    const int W = 2 * span + 1;
    hipLaunchKernelGGL(bias_expand_kernel, dim3((unsigned)((W * W + kThreads - 1) / kThreads), (unsigned)H),
                       dim3(kThreads), 0, stream, table, lut, nb, W, H, dt, bias);
    return hipGetLastError();
}

hipError_t launch_bias_gradient(const float* dbias, const int32_t* lut, int nb, int span, int H, int dt, void* dtable,
                                hipStream_t stream)
{
    hipLaunchKernelGGL(bias_gradient_kernel, dim3((unsigned)nb, (unsigned)H), dim3(kMaxWidth), 0, stream, dbias, lut,
                       nb, 2 * span + 1, H, dt, dtable);
    return hipGetLastError();
}

}  // namespace mpm

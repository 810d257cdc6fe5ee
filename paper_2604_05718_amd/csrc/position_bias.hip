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

// dtable[bucket][h] = sum of dbias[h] over the bucket's offsets, in the order of the offsets: one
// wave a bucket and head. Row offsets are scanned for the row bucket; in a row that has it,
// lanes take columns lane, lane + 64, ... and those of the column bucket are added; a butterfly
// joins the lanes, so the order is the same on every run.
__global__ __launch_bounds__(kThreads) void bias_gradient_kernel(const float* __restrict__ dbias,
                                                                 const int32_t* __restrict__ lut, int nb, int W, int H,
                                                                 int dt, void* __restrict__ dtable)
{
    __shared__ int32_t axis[256];
    if (threadIdx.x < W) axis[threadIdx.x] = lut[threadIdx.x];
    __syncthreads();
    const int lane = threadIdx.x % kWave;
    const long item = (long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
    if (item >= (long)nb * nb * H) return;
    const int h = (int)(item % H), bucket = (int)(item / H), br = bucket / nb, bc = bucket % nb;
    float sum = 0.0f;
    for (int r = 0; r < W; ++r) {
        if (axis[r] != br) continue;
        for (int c = lane; c < W; c += kWave)
            if (axis[c] == bc) sum += dbias[((long)h * W + r) * W + c];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane != 0) return;
    if (dt == kBf16) reinterpret_cast<uint16_t*>(dtable)[item] = (uint16_t)f32_to_bf16_rne(sum);
    else reinterpret_cast<float*>(dtable)[item] = sum;
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
    const long items = (long)nb * nb * H;
    const int per = kThreads / kWave;
    hipLaunchKernelGGL(bias_gradient_kernel, dim3((unsigned)((items + per - 1) / per)), dim3(kThreads), 0, stream,
                       dbias, lut, nb, 2 * span + 1, H, dt, dtable);
    return hipGetLastError();
}

}  // namespace mpm

// Zeros in the rows of no image of up to three tensors of rows of heads: those before off[0] and from off[B] on. Usually
// there are none and the launch is all it costs (2 us).
#include <algorithm>

#include "mpm_device.h"
#include "mpm_launch.h"

namespace mpm {
namespace {

constexpr int kThreads = 256;
constexpr int kMost = 3;

struct Clears {
    ClearRows c[kMost];
    int vecs[kMost];  // of a row
};

__global__ __launch_bounds__(kThreads) void clear_rows_kernel(Clears all, int dh_vecs, int bytes)
{
    const ClearRows c = all.c[blockIdx.y];
    const int vecs = all.vecs[blockIdx.y];
    const long lo = min(max((long)c.off[0], 0L), c.R), hi = min(max((long)c.off[c.B], lo), c.R), many = lo + c.R - hi;
    const u32x4 none = {0, 0, 0, 0};
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < many * vecs; i += (long)gridDim.x * kThreads) {
        const long r = i / vecs;
        const int v = (int)(i - r * vecs), head = v / dh_vecs;
        const long row = r < lo ? r : r - lo + hi;
        store16(c.x.p + (row * c.x.row + head * c.x.head) * bytes + (v - head * dh_vecs) * 16L, none);
    }
}

}  // namespace

hipError_t launch_clear_rows(const ClearRows* c, int n, int dh, int dt, hipStream_t stream)
{
    const int bytes = dt == kBf16 ? 2 : 4, dh_vecs = dh * bytes / 16;
    Clears all{};
    long most = 0;
    for (int i = 0; i < n; ++i) {
        all.c[i] = c[i];
        all.vecs[i] = c[i].H * dh_vecs;
        most = std::max(most, c[i].R * all.vecs[i]);
    }
    hipLaunchKernelGGL(clear_rows_kernel, dim3((unsigned)std::min(256L, (most + kThreads - 1) / kThreads), (unsigned)n),
                       dim3(kThreads), 0, stream, all, dh_vecs, bytes);
    return hipGetLastError();
}

}  // namespace mpm

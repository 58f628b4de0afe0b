// Group norm with residual and activation over NHWC maps (layers of the forward pass of a served network, paper Sec. 5):
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c] + r)
// with mean and var over the H x W x C / groups values of an image's group of channels.  Statistics are in fp32, the
// variance as the mean square of the differences from the mean (not of the values, which loses it where the mean is large).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act_device.h"
#include "device_util.h"
#include "gpulet_internal.h"

namespace gpulet {
namespace {

struct Params {
    const void *x, *r;
    const float *gamma, *beta;
    void *y;
    int C, HW, G, cg, ldx, ldr, ldy, act;
    float eps;
};

template <int T>
__device__ __forceinline__ float block_sum(float v, float *lds) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) s += lds[i];
    return s;
}

// One workgroup per image and group.
template <typename T>
__global__ __launch_bounds__(256) void group_norm_kernel(Params p) {
    __shared__ float lds[4];
    const int n = blockIdx.x / p.G, g = blockIdx.x - n * p.G;
    const long long px = static_cast<long long>(n) * p.HW;
    const T *x = static_cast<const T *>(p.x) + px * p.ldx + g * p.cg;
    const int count = p.HW * p.cg;
    float s = 0.f;
    for (int i = threadIdx.x; i < count; i += 256) {
        const int q = i / p.cg, c = i - q * p.cg;
        s += static_cast<float>(x[q * p.ldx + c]);
    }
    const float mean = block_sum<256>(s, lds) / static_cast<float>(count);
    s = 0.f;
    for (int i = threadIdx.x; i < count; i += 256) {
        const int q = i / p.cg, c = i - q * p.cg;
        const float d = static_cast<float>(x[q * p.ldx + c]) - mean;
        s += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum<256>(s, lds) / static_cast<float>(count) + p.eps);
    const T *r = p.r ? static_cast<const T *>(p.r) + px * p.ldr + g * p.cg : nullptr;
    T *y = static_cast<T *>(p.y) + px * p.ldy + g * p.cg;
    for (int i = threadIdx.x; i < count; i += 256) {
        const int q = i / p.cg, c = i - q * p.cg;
        float v[1] = {(static_cast<float>(x[q * p.ldx + c]) - mean) * rstd};
        if (p.gamma) v[0] *= p.gamma[g * p.cg + c];
        if (p.beta) v[0] += p.beta[g * p.cg + c];
        if (r) v[0] += static_cast<float>(r[q * p.ldr + c]);
        activate(v, p.act);
        y[q * p.ldy + c] = static_cast<T>(v[0]);
    }
}

}  // namespace

hipError_t launch_group_norm(const GroupNormArgs &a, const LaunchCtx &ctx, hipStream_t stream) {
    Params p{};
    p.x = a.x; p.r = a.residual; p.gamma = a.gamma; p.beta = a.beta; p.y = a.y;
    p.C = a.C; p.HW = a.H * a.W; p.G = a.groups; p.cg = a.C / a.groups;
    p.ldx = a.ldx; p.ldr = a.ldr; p.ldy = a.ldy;
    p.act = a.act; p.eps = a.eps;
    const dim3 grid(a.N * a.groups);
    if (a.dtype == GPULET_BF16) group_norm_kernel<__bf16><<<grid, 256, 0, stream>>>(p);
    else if (a.dtype == GPULET_F16) group_norm_kernel<_Float16><<<grid, 256, 0, stream>>>(p);
    else group_norm_kernel<float><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

size_t group_norm_workspace(const GroupNormArgs &a) { return 0; }

}  // namespace gpulet

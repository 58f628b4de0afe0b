// Matrix product with bias, residual and activation in its epilogue on gfx950 matrix cores:
//   y[m, n] = act(sum_k x[m, k] w[n, k] + b[n] + r[m, n])
// for the per-pixel and per-row layers of a forward pass (paper Sec. 5) that a ReLU convolution or the fully connected
// layer cannot stand for: wide activations, fp16, fp32 results, rows that are slices of wider ones, any number of rows.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act_device.h"
#include "device_util.h"
#include "gpulet_internal.h"

namespace gpulet {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ __forceinline__ f32x4 mma(const uint4 &a, const uint4 &b, const f32x4 c, __bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8 *>(&a), *reinterpret_cast<const bf16x8 *>(&b),
                                                   c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const uint4 &a, const uint4 &b, const f32x4 c, _Float16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8 *>(&a), *reinterpret_cast<const f16x8 *>(&b),
                                                  c, 0, 0, 0);
}

struct Params {
    const void *x, *w;
    const float *b;
    const void *r;
    void *y;
    int M, N, K, ldx, ldw, ldr, ldy, act;
    int tiles_n;
    FastDiv d_tiles_n;
};

// bias, residual and activation on N consecutive columns of row m, then the store.
template <int N, typename T, ActCode A>
__device__ __forceinline__ void finish(const Params &p, int m, int n, float (&v)[N]) {
    const T *r = p.r ? static_cast<const T *>(p.r) + static_cast<long long>(m) * p.ldr + n : nullptr;
    T *y = static_cast<T *>(p.y) + static_cast<long long>(m) * p.ldy + n;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (n + i >= p.N) break;
        if (p.b) v[i] += p.b[n + i];
        if (r) v[i] += static_cast<float>(r[i]);
    }
    activate<A>(v, p.act);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (n + i < p.N) y[i] = static_cast<T>(v[i]);
}

// Elements [k, k + 8) of a row; zero past its end.  Rows may start at any element.
template <typename T>
__device__ __forceinline__ uint4 load8(const T *row, int k, int K, bool row_ok) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (!row_ok || k >= K) return v;
    if (k + 8 <= K) {
        __builtin_memcpy(&v, row + k, 16);
        return v;
    }
    unsigned short e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k + i < K ? reinterpret_cast<const unsigned short *>(row)[k + i] : 0;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// A tile of 64 rows by 64 columns a workgroup, four wavefronts of 32 x 32, one slice of 64 elements of the depth at a time
// through LDS, the next one on its way into registers meanwhile.  Takes any alignment and any depth.
template <typename T, typename TO, ActCode A>
__global__ __launch_bounds__(256) void matmul_any_kernel(Params p) {
    __shared__ uint4 tile[2][64 * 8];   // x and w: 64 rows of 8 chunks of 8 elements
    const int tm = fdiv(blockIdx.x, p.d_tiles_n), tn = blockIdx.x - tm * p.tiles_n;
    const int m0 = tm * 64, n0 = tn * 64;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const int q = threadIdx.x & 7, row = threadIdx.x >> 3;   // a thread stages chunk q of rows row and row + 32
    const T *xr[2], *wr[2];
    bool xok[2], wok[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int m = m0 + row + 32 * i, n = n0 + row + 32 * i;
        xok[i] = m < p.M;
        wok[i] = n < p.N;
        xr[i] = static_cast<const T *>(p.x) + static_cast<long long>(xok[i] ? m : 0) * p.ldx;
        wr[i] = static_cast<const T *>(p.w) + static_cast<long long>(wok[i] ? n : 0) * p.ldw;
    }
    uint4 xs[2], ws[2];
    auto fetch = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            xs[i] = load8(xr[i], k + 8 * q, p.K, xok[i]);
            ws[i] = load8(wr[i], k + 8 * q, p.K, wok[i]);
        }
    };
    f32x4 acc[2][2] = {};
    fetch(0);
    for (int k = 0; k < p.K; k += 64) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = (row + 32 * i) * 8 + (q ^ ((row >> 1) & 7));
            tile[0][at] = xs[i];
            tile[1][at] = ws[i];
        }
        __syncthreads();
        if (k + 64 < p.K) fetch(k + 64);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint4 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int rw = 16 * i + (lane & 15), c = (4 * h + (lane >> 4)) ^ ((rw >> 1) & 7);
                a[i] = tile[1][(wn + rw) * 8 + c];
                b[i] = tile[0][(wm + rw) * 8 + c];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = mma(a[j], b[i], acc[i][j], T());
        }
    }
    // w is the left operand: a lane holds four consecutive columns of one row of y
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int m = m0 + wm + 16 * i + (lane & 15), n = n0 + wn + 16 * j + 4 * (lane >> 4);
            float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (m < p.M && n < p.N) finish<4, TO, A>(p, m, n, v);
        }
}

template <typename T, typename TO>
hipError_t launch_any(const Params &p, int tiles_m, hipStream_t stream) {
    const dim3 grid(tiles_m * p.tiles_n);
    switch (act_code(p.act)) {
        case ActCode::NORMAL: matmul_any_kernel<T, TO, ActCode::NORMAL><<<grid, 256, 0, stream>>>(p); break;
        case ActCode::GATE: matmul_any_kernel<T, TO, ActCode::GATE><<<grid, 256, 0, stream>>>(p); break;
        default: matmul_any_kernel<T, TO, ActCode::LINEAR><<<grid, 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul(const MatmulArgs &a, const LaunchCtx &ctx, hipStream_t stream) {
    Params p{};
    p.x = a.x; p.w = a.w; p.b = a.b; p.r = a.residual; p.y = a.y;
    p.M = a.M; p.N = a.N; p.K = a.K;
    p.ldx = a.ldx; p.ldw = a.ldw; p.ldr = a.ldr; p.ldy = a.ldy;
    p.act = a.act;
    p.tiles_n = (a.N + 63) / 64;
    p.d_tiles_n = make_fastdiv(p.tiles_n);
    const int tiles_m = (a.M + 63) / 64;
    if (a.dtype == GPULET_BF16)
        return a.out_dtype == GPULET_F32 ? launch_any<__bf16, float>(p, tiles_m, stream) : launch_any<__bf16, __bf16>(p, tiles_m, stream);
    return a.out_dtype == GPULET_F32 ? launch_any<_Float16, float>(p, tiles_m, stream) : launch_any<_Float16, _Float16>(p, tiles_m, stream);
}

size_t matmul_workspace(const MatmulArgs &a) { return 0; }

}  // namespace gpulet

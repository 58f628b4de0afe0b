// Single-layer entry points of the C ABI: argument checks, then a launch on
// the caller's stream (paper Sec. 5: the executor runs the model's layers on
// its gpu-let).
#include <cstdint>
#include <initializer_list>

#include "gpulet_internal.h"

using namespace gpulet;

namespace {

gpulet_status make_conv_args(ConvArgs &a, const void *x, const void *w, const float *b, void *y,
                             int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                             int relu, const void *residual, int y_ch_stride, int y_ch_offset) {
    a.x = x; a.w = w; a.b = b; a.y = y; a.residual = residual;
    a.N = N; a.C = C; a.H = H; a.W = W; a.K = K; a.R = R; a.S = S;
    a.stride = stride; a.pad = pad; a.relu = relu ? 1 : 0;
    a.y_ch_stride = y_ch_stride == 0 ? K : y_ch_stride;
    a.y_ch_offset = y_ch_offset;
    if (stride < 1 || R < 1 || S < 1 || pad < 0 || H < 1 || W < 1) return GPULET_EINVAL;
    a.P = out_extent(H, R, stride, pad);
    a.Q = out_extent(W, S, stride, pad);
    return check_conv(a);
}

// `rows` rows of `width` bytes, `pitch` bytes apart.
struct Rows {
    uintptr_t at;
    uint64_t rows, width, pitch;
    uint64_t span() const { return rows ? (rows - 1) * pitch + width : 0; }
};
Rows make_rows(const void *p, uint64_t rows, uint64_t width, uint64_t pitch) {
    return Rows{reinterpret_cast<uintptr_t>(p), p ? rows : 0, width, pitch};
}

// Whether the two share a byte.  Slices of the same wide rows (equal pitches) are compared by their columns; rows of
// different pitches count as sharing where their address ranges meet.
bool meet(const Rows &a, const Rows &b) {
    if (a.span() == 0 || b.span() == 0) return false;
    if (a.at >= b.at + b.span() || b.at >= a.at + a.span()) return false;
    if (a.pitch != b.pitch) return true;
    const uint64_t d = a.at <= b.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;
    // in a's frame a covers columns [0, a.width), b covers [d, d + b.width), wrapping into the next row
    return d < a.width || d + b.width > a.pitch;
}

gpulet_status check_workspace(const void *ws, size_t bytes) {
    return bytes > 0 && ws && reinterpret_cast<uintptr_t>(ws) % 256 != 0 ? GPULET_EINVAL : GPULET_OK;
}

constexpr int kMaxRow = 1 << 20;   // elements: 256 rows of fp32 stay below 2^31 bytes

int type_bytes(int t) { return t == GPULET_F32 ? 4 : 2; }
bool misaligned(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(bytes) != 0; }

}  // namespace

namespace gpulet {

gpulet_status check_matmul(const gpulet_matmul_desc *d, MatmulArgs &a) {
    if (!d || !d->x || !d->w || !d->y) return GPULET_EINVAL;
    if (d->M < 1 || d->N < 1 || d->K < 1 || d->M > (1 << 24) || d->N > kMaxRow || d->K > kMaxRow) return GPULET_EINVAL;
    if ((d->M + 63LL) / 64 * ((d->N + 63LL) / 64) > (1 << 23)) return GPULET_EINVAL;
    if (d->dtype != GPULET_BF16 && d->dtype != GPULET_F16) return GPULET_EINVAL;
    if (d->out_dtype != d->dtype && d->out_dtype != GPULET_F32) return GPULET_EINVAL;
    if (d->act < GPULET_ACT_NONE || d->act > GPULET_ACT_GELU_TANH) return GPULET_EINVAL;
    a = MatmulArgs{d->x, d->w, d->b, d->residual, d->y, d->M, d->N, d->K, d->ldx ? d->ldx : d->K, d->ldw ? d->ldw : d->K,
                   d->ldr ? d->ldr : d->N, d->ldy ? d->ldy : d->N, d->dtype, d->out_dtype, d->act, nullptr, 0};
    if (a.ldx < a.K || a.ldw < a.K || a.ldr < a.N || a.ldy < a.N) return GPULET_EINVAL;
    if (a.ldx > kMaxRow || a.ldw > kMaxRow || a.ldr > kMaxRow || a.ldy > kMaxRow) return GPULET_EINVAL;
    const int es = type_bytes(a.out_dtype);
    if (misaligned(a.x, 2) || misaligned(a.w, 2) || misaligned(a.b, 4) || misaligned(a.residual, es) || misaligned(a.y, es))
        return GPULET_EINVAL;
    const uint64_t M = a.M, N = a.N, K = a.K;
    const Rows y = make_rows(a.y, M, es * N, 1ull * es * a.ldy), r = make_rows(a.residual, M, es * N, 1ull * es * a.ldr);
    if (meet(y, make_rows(a.x, M, 2 * K, 2ull * a.ldx)) || meet(y, make_rows(a.w, N, 2 * K, 2ull * a.ldw)) ||
        meet(y, make_rows(a.b, 1, 4 * N, 4 * N)))
        return GPULET_EINVAL;
    if (!(a.residual == a.y && a.ldr == a.ldy) && meet(y, r)) return GPULET_EINVAL;
    return GPULET_OK;
}

gpulet_status check_group_norm(const gpulet_group_norm_desc *d, GroupNormArgs &a) {
    if (!d || !d->x || !d->y) return GPULET_EINVAL;
    if (d->N < 1 || d->C < 1 || d->H < 1 || d->W < 1 || d->groups < 1 || d->C % d->groups != 0) return GPULET_EINVAL;
    if (d->dtype < GPULET_BF16 || d->dtype > GPULET_F32 || d->act < GPULET_ACT_NONE || d->act > GPULET_ACT_GELU_TANH)
        return GPULET_EINVAL;
    if (!(d->eps >= 0.f) || d->eps > 3.0e38f) return GPULET_EINVAL;
    if (1LL * d->N * d->groups > (1 << 21)) return GPULET_EINVAL;
    a = GroupNormArgs{d->x, d->gamma, d->beta, d->residual, d->y, d->N, d->C, d->H, d->W, d->groups,
                      d->x_ch_stride ? d->x_ch_stride : d->C, d->r_ch_stride ? d->r_ch_stride : d->C,
                      d->y_ch_stride ? d->y_ch_stride : d->C, d->dtype, d->act, d->eps, nullptr, 0};
    if (a.ldx < a.C || a.ldr < a.C || a.ldy < a.C) return GPULET_EINVAL;
    const int es = type_bytes(a.dtype);
    const long long px = 1LL * a.H * a.W;
    for (int ld : {a.ldx, a.ldr, a.ldy})
        if (px >= (1LL << 31) || px * ld >= (1LL << 31) / es) return GPULET_EINVAL;
    if (misaligned(a.x, es) || misaligned(a.residual, es) || misaligned(a.y, es) || misaligned(a.gamma, 4) || misaligned(a.beta, 4))
        return GPULET_EINVAL;
    const uint64_t all = 1ull * a.N * px, C = a.C;
    const Rows y = make_rows(a.y, all, es * C, 1ull * es * a.ldy);
    if (meet(y, make_rows(a.gamma, 1, 4 * C, 4 * C)) || meet(y, make_rows(a.beta, 1, 4 * C, 4 * C))) return GPULET_EINVAL;
    if (!(a.x == a.y && a.ldx == a.ldy) && meet(y, make_rows(a.x, all, es * C, 1ull * es * a.ldx))) return GPULET_EINVAL;
    if (!(a.residual == a.y && a.ldr == a.ldy) && meet(y, make_rows(a.residual, all, es * C, 1ull * es * a.ldr)))
        return GPULET_EINVAL;
    // a thread has nearly an element at least
    if (all * C > (1ull << 30) && !group_norm_fits(a)) return GPULET_EINVAL;
    return GPULET_OK;
}

}  // namespace gpulet

extern "C" gpulet_status gpulet_matmul_workspace_bytes(const gpulet_matmul_desc *d, size_t *bytes) {
    if (!bytes) return GPULET_EINVAL;
    MatmulArgs a;
    const gpulet_status st = check_matmul(d, a);
    if (st == GPULET_OK) *bytes = matmul_workspace(a);
    return st;
}

extern "C" gpulet_status gpulet_matmul(const gpulet_matmul_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
    MatmulArgs a;
    gpulet_status st = check_matmul(d, a);
    if (st == GPULET_OK && workspace) {
        a.ws = workspace;
        a.ws_bytes = workspace_bytes;
        st = check_workspace(workspace, workspace_bytes);
        const int es = type_bytes(a.out_dtype);
        const Rows ws = make_rows(workspace, 1, workspace_bytes, workspace_bytes);
        if (meet(ws, make_rows(a.x, a.M, 2ull * a.K, 2ull * a.ldx)) || meet(ws, make_rows(a.w, a.N, 2ull * a.K, 2ull * a.ldw)) ||
            meet(ws, make_rows(a.b, 1, 4ull * a.N, 4ull * a.N)) ||
            meet(ws, make_rows(a.residual, a.M, 1ull * es * a.N, 1ull * es * a.ldr)) ||
            meet(ws, make_rows(a.y, a.M, 1ull * es * a.N, 1ull * es * a.ldy)))
            return GPULET_EINVAL;
    }
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_matmul(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_group_norm_workspace_bytes(const gpulet_group_norm_desc *d, size_t *bytes) {
    if (!bytes) return GPULET_EINVAL;
    GroupNormArgs a;
    const gpulet_status st = check_group_norm(d, a);
    if (st == GPULET_OK) *bytes = group_norm_workspace(a);
    return st;
}

extern "C" gpulet_status gpulet_group_norm(const gpulet_group_norm_desc *d, void *workspace, size_t workspace_bytes,
                                           void *stream) {
    GroupNormArgs a;
    gpulet_status st = check_group_norm(d, a);
    if (st != GPULET_OK) return st;
    const size_t need = group_norm_workspace(a);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return GPULET_ENOMEM;
        st = check_workspace(workspace, workspace_bytes);
        if (st != GPULET_OK) return st;
        const uint64_t all = 1ull * a.N * a.H * a.W, es = static_cast<uint64_t>(type_bytes(a.dtype));
        const Rows ws = make_rows(workspace, 1, need, need);
        if (meet(ws, make_rows(a.x, all, es * a.C, es * a.ldx)) || meet(ws, make_rows(a.residual, all, es * a.C, es * a.ldr)) ||
            meet(ws, make_rows(a.y, all, es * a.C, es * a.ldy)) || meet(ws, make_rows(a.gamma, 1, 4ull * a.C, 4ull * a.C)) ||
            meet(ws, make_rows(a.beta, 1, 4ull * a.C, 4ull * a.C)))
            return GPULET_EINVAL;
        a.ws = workspace;
        a.ws_bytes = workspace_bytes;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_group_norm(a, s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv2d_fwd_ex(const void *x, const void *w, const float *b, void *y,
                                              int N, int C, int H, int W, int K, int R, int S,
                                              int stride, int pad, int relu, const void *residual,
                                              int y_ch_stride, int y_ch_offset, void *stream) {
    ConvArgs a;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, R, S, stride, pad, relu, residual,
                                      y_ch_stride, y_ch_offset);
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv2d_fwd_slices(const void *x, const void *w, const float *b, void *y, int N,
                                                  int C, int H, int W, int K, int R, int S, int stride,
                                                  int pad, int relu, const void *residual, int x_ch_stride,
                                                  int x_ch_offset, int y_ch_stride, int y_ch_offset,
                                                  void *stream) {
    ConvArgs a;
    a.x_ch_stride = x_ch_stride;
    a.x_ch_offset = x_ch_offset;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, R, S, stride, pad, relu, residual,
                                      y_ch_stride, y_ch_offset);
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv1x1_fwd_two_outputs(const void *x, const void *w, const float *b, void *y,
                                                        void *y2, int N, int C, int H, int W, int K, int k2,
                                                        int stride, int relu, int x_ch_stride, int x_ch_offset,
                                                        int y_ch_stride, int y_ch_offset, int y2_ch_stride,
                                                        int y2_ch_offset, void *stream) {
    if (!y2 || k2 < 1 || k2 >= K) return GPULET_EINVAL;
    ConvArgs a;
    a.x_ch_stride = x_ch_stride;
    a.x_ch_offset = x_ch_offset;
    a.y2 = y2;
    a.k2 = k2;
    a.y2_ch_stride = y2_ch_stride == 0 ? K - k2 : y2_ch_stride;
    a.y2_ch_offset = y2_ch_offset;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, 1, 1, stride, 0, relu, nullptr,
                                      y_ch_stride == 0 ? k2 : y_ch_stride, y_ch_offset);
    if (st != GPULET_OK) return st;
    const int ldx = x_ch_stride ? x_ch_stride : C;
    if (C % 8 != 0 || ldx % 8 != 0 || x_ch_offset % 8 != 0 || reinterpret_cast<uintptr_t>(x) % 16 != 0 ||
        reinterpret_cast<uintptr_t>(w) % 16 != 0)
        return GPULET_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv2d_group_fwd(const gpulet_conv_desc *layers, int n, void *stream) {
    if (!layers || n < 1 || n > kMaxGroup) return GPULET_EINVAL;
    ConvArgs a[kMaxGroup];
    struct Range { uintptr_t lo, hi; };
    Range xr[kMaxGroup], rr[kMaxGroup], yr[kMaxGroup];
    for (int j = 0; j < n; ++j) {
        const gpulet_conv_desc &d = layers[j];
        a[j].x_ch_stride = d.x_ch_stride;
        a[j].x_ch_offset = d.x_ch_offset;
        gpulet_status st = make_conv_args(a[j], d.x, d.w, d.b, d.y, d.N, d.C, d.H, d.W, d.K, d.R, d.S, d.stride,
                                          d.pad, d.relu, d.residual, d.y_ch_stride, d.y_ch_offset);
        if (st != GPULET_OK) return st;
        const uintptr_t ldx = static_cast<uintptr_t>(d.x_ch_stride ? d.x_ch_stride : d.C);
        const uintptr_t px = static_cast<uintptr_t>(d.N) * d.H * d.W, py = static_cast<uintptr_t>(d.N) * a[j].P * a[j].Q;
        xr[j] = {reinterpret_cast<uintptr_t>(d.x), reinterpret_cast<uintptr_t>(d.x) + 2 * px * ldx};
        rr[j] = {reinterpret_cast<uintptr_t>(d.residual),
                 d.residual ? reinterpret_cast<uintptr_t>(d.residual) + 2 * py * d.K : 0};
        yr[j] = {reinterpret_cast<uintptr_t>(d.y), reinterpret_cast<uintptr_t>(d.y) + 2 * py * a[j].y_ch_stride};
    }
    auto meet = [](const Range &p, const Range &q) { return p.lo < q.hi && q.lo < p.hi; };
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j) {
            if (i == j) continue;
            if (meet(yr[i], xr[j]) || (rr[j].hi && meet(yr[i], rr[j]))) return GPULET_EINVAL;
            if (i < j && meet(yr[i], yr[j])) {
                // only as disjoint channel slices of one tensor
                const bool slices = a[i].y == a[j].y && a[i].y_ch_stride == a[j].y_ch_stride && a[i].P == a[j].P &&
                                    a[i].Q == a[j].Q && a[i].N == a[j].N &&
                                    (a[i].y_ch_offset + a[i].K <= a[j].y_ch_offset ||
                                     a[j].y_ch_offset + a[j].K <= a[i].y_ch_offset);
                if (!slices) return GPULET_EINVAL;
            }
        }
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv_group(a, n, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv1x1_maxpool3_fwd(const void *x, const void *w, const float *b, void *y,
                                                     void *y2, void *pool_y, int N, int C, int H, int W, int K,
                                                     int k2, int relu, int y_ch_stride, int y_ch_offset,
                                                     int y2_ch_stride, int y2_ch_offset, void *stream) {
    if (!pool_y || reinterpret_cast<uintptr_t>(pool_y) % 16 != 0) return GPULET_EINVAL;
    if (y2 && (k2 < 1 || k2 >= K)) return GPULET_EINVAL;
    ConvArgs a;
    a.pool_y = pool_y;
    const int k1 = y2 ? k2 : K;
    if (y2) {
        a.y2 = y2;
        a.k2 = k2;
        a.y2_ch_stride = y2_ch_stride == 0 ? K - k2 : y2_ch_stride;
        a.y2_ch_offset = y2_ch_offset;
    }
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, 1, 1, 1, 0, relu, nullptr,
                                      y_ch_stride == 0 ? k1 : y_ch_stride, y_ch_offset);
    if (st != GPULET_OK) return st;
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0 || reinterpret_cast<uintptr_t>(w) % 16 != 0) return GPULET_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_maxpool3_conv1x1_fwd(const void *x, const void *w, const float *b, void *y, int N,
                                                     int C, int H, int W, int K, int relu, int y_ch_stride,
                                                     int y_ch_offset, void *stream) {
    ConvArgs a;
    a.pre_pool = 3;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, 1, 1, 1, 0, relu, nullptr, y_ch_stride,
                                      y_ch_offset);
    if (st != GPULET_OK) return st;
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0 || reinterpret_cast<uintptr_t>(w) % 16 != 0) return GPULET_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv3x3_maxpool2_fwd(const void *x, const void *w, const float *b, void *y, int N,
                                                     int C, int H, int W, int K, int y_ch_stride, int y_ch_offset,
                                                     void *stream) {
    ConvArgs a;
    a.post_pool2 = 2;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, 3, 3, 1, 1, 1, nullptr, y_ch_stride, y_ch_offset);
    if (st != GPULET_OK) return st;
    // what the kernel with the pooled epilogue needs: whole 64-channel blocks, 16-byte stores
    if (C % 64 != 0 || K % 8 != 0 || a.y_ch_stride % 8 != 0 || a.y_ch_offset % 8 != 0 ||
        reinterpret_cast<uintptr_t>(x) % 16 != 0 || reinterpret_cast<uintptr_t>(w) % 16 != 0 ||
        reinterpret_cast<uintptr_t>(y) % 16 != 0 || reinterpret_cast<uintptr_t>(b) % 16 != 0)
        return GPULET_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_conv(a, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_set_conv_pool_fusion(int on) {
    if (on != 0 && on != 1) return GPULET_EINVAL;
    set_conv_pool_fusion(on);
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_conv2d_fwd(const void *x, const void *w, const float *b, void *y,
                                           int N, int C, int H, int W, int K, int R, int S,
                                           int stride, int pad, int relu, void *stream) {
    return gpulet_conv2d_fwd_ex(x, w, b, y, N, C, H, W, K, R, S, stride, pad, relu, nullptr, 0, 0,
                                stream);
}

extern "C" gpulet_status gpulet_conv2d_timeline(const void *x, const void *w, const float *b, void *y, int N, int C,
                                                int H, int W, int K, int R, int S, int stride, int pad, int relu,
                                                void *stream, int warmup, int64_t *stamps, int *workgroups) {
    if (!stamps || !workgroups || warmup < 0) return GPULET_EINVAL;
    ConvArgs a;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, R, S, stride, pad, relu, nullptr, 0, 0);
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const LaunchCtx ctx = stream_ctx(s);
    constexpr size_t kBytes = 8 * 8 * sizeof(int64_t);
    void *dev = nullptr;
    GPULET_HIP(hipMalloc(&dev, kBytes));
    hipError_t e = hipMemsetAsync(dev, 0, kBytes, s);
    for (int i = 0; i < warmup && e == hipSuccess; ++i) e = launch_conv(a, ctx, s);
    a.stamps = dev;
    if (e == hipSuccess) e = launch_conv(a, ctx, s);
    if (e == hipSuccess) e = hipMemcpyAsync(stamps, dev, kBytes, hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    (void)hipFree(dev);
    if (e != hipSuccess) return hip_fail(e);
    int n = 0;
    while (n < 8 && stamps[n * 8] != 0) ++n;
    *workgroups = n;
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_set_conv_tile(int tile) {
    if (tile < -1 || tile >= GPULET_CONV_TILES) return GPULET_EINVAL;
    set_conv_tile(tile);
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_set_conv_split_k(int max_split) {
    if (max_split < 1 || max_split > 8) return GPULET_EINVAL;
    set_conv_split_k(max_split);
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_depthwise_conv2d_fwd(const void *x, const void *w, const float *b, void *y,
                                                     int N, int C, int H, int W, int R, int S, int stride,
                                                     int pad, int relu, void *stream) {
    if (!x || !w || !y) return GPULET_EINVAL;
    int P = 0, Q = 0;
    gpulet_status st = check_dwconv(N, C, H, W, R, S, stride, pad, &P, &Q);
    if (st != GPULET_OK) return st;
    GPULET_HIP(launch_dwconv(x, w, b, y, N, C, H, W, R, S, stride, pad, relu ? 1 : 0, P, Q,
                             static_cast<hipStream_t>(stream)));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_pool(const void *x, void *y, int N, int C, int H, int W, int mode,
                                     int k, int stride, int pad, void *stream) {
    if (!x || !y) return GPULET_EINVAL;
    int P = 0, Q = 0;
    gpulet_status st = check_pool(N, C, H, W, mode, k, stride, pad, &P, &Q);
    if (st != GPULET_OK) return st;
    GPULET_HIP(launch_pool(x, y, N, C, H, W, P, Q, mode, k, stride, pad, static_cast<hipStream_t>(stream)));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_fc(const void *x, const void *w, const float *b, void *y, int N,
                                   int In, int Out, int relu, int out_fp32, void *stream) {
    if (!x || !w || !y) return GPULET_EINVAL;
    gpulet_status st = check_fc(N, In, Out);
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    GPULET_HIP(launch_fc(x, w, b, y, N, In, Out, relu ? 1 : 0, out_fp32 ? 1 : 0, stream_ctx(s), s));
    return GPULET_OK;
}

extern "C" gpulet_status gpulet_fc_static_scratch(const void *x, const void *w, const float *b, void *y, int N,
                                                  int In, int Out, int relu, int out_fp32, void *stream) {
    if (!x || !w || !y) return GPULET_EINVAL;
    gpulet_status st = check_fc(N, In, Out);
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    bool too_large = false;
    GPULET_HIP(launch_fc_static(x, w, b, y, N, In, Out, relu ? 1 : 0, out_fp32 ? 1 : 0, stream_ctx(s).n_cu, s,
                                &too_large));
    return too_large ? GPULET_ENOMEM : GPULET_OK;
}

extern "C" gpulet_status gpulet_time_conv2d(const void *x, const void *w, const float *b, void *y,
                                            int N, int C, int H, int W, int K, int R, int S,
                                            int stride, int pad, int relu, const void *residual,
                                            int y_ch_stride, int y_ch_offset, void *stream,
                                            int warmup, int iters, float *avg_ms) {
    if (!avg_ms || iters < 1 || warmup < 0) return GPULET_EINVAL;
    ConvArgs a;
    gpulet_status st = make_conv_args(a, x, w, b, y, N, C, H, W, K, R, S, stride, pad, relu, residual,
                                      y_ch_stride, y_ch_offset);
    if (st != GPULET_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const LaunchCtx ctx = stream_ctx(s);
    for (int i = 0; i < warmup; ++i) GPULET_HIP(launch_conv(a, ctx, s));
    hipEvent_t e0 = nullptr, e1 = nullptr;
    GPULET_HIP(hipEventCreate(&e0));
    hipError_t e = hipEventCreate(&e1);
    if (e != hipSuccess) {
        (void)hipEventDestroy(e0);
        return hip_fail(e);
    }
    e = hipEventRecord(e0, s);
    for (int i = 0; i < iters && e == hipSuccess; ++i) e = launch_conv(a, ctx, s);
    if (e == hipSuccess) e = hipEventRecord(e1, s);
    if (e == hipSuccess) e = hipEventSynchronize(e1);
    float ms = 0.f;
    if (e == hipSuccess) e = hipEventElapsedTime(&ms, e0, e1);
    (void)hipEventDestroy(e0);
    (void)hipEventDestroy(e1);
    if (e != hipSuccess) return hip_fail(e);
    *avg_ms = ms / static_cast<float>(iters);
    return GPULET_OK;
}

// Group norm with residual and activation over NHWC maps (layers of the forward pass of a served network, paper Sec. 5):
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c] + r)
// with mean and var over the H x W x C / groups values of an image's group of channels.  Statistics are in fp32, the
// variance as the mean square of the differences from a mean (not of the values, which loses it where the mean is large).
//
// Bound by memory: x is read once and y written once, with about 20 vector operations an element.  Two forms:
//
// * held: a workgroup keeps whole groups of one image in registers: one launch, x read once.  For groups of up to
//   kHeldBytes.
// * two launches for larger groups: the first reduces chunks of an image to (mean, sum of squared differences) per group,
//   the second joins them and reads x again.
//
// Which one runs depends on the shape of an image and the alignment of its rows only, not on how many images there are or
// on the CUs of the gpu-let, so that an image's result has the same bits in any batch.
//
// A thread handles units of V consecutive channels of one group (V the largest power of two that divides the group and keeps
// all tensors' rows aligned, 16 bytes at most) and keeps its channels from pixel to pixel, so that its scale and shift stay
// in registers; the threads of a workgroup cover consecutive units of a pixel, then the next pixel.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act_device.h"
#include "device_util.h"
#include "gpulet_internal.h"

namespace gpulet {
namespace {

constexpr unsigned OOB = 0x80000000u;   // byte offset past every image: loads give zero, stores do nothing
constexpr int kMaxThreads = 1024;
constexpr int kMaxGb = 64;              // groups of a workgroup at most

struct Params {
    const void *x, *r;
    const float *gamma, *beta;
    void *y;
    float2 *part;             // two launches: [image][group][chunk] (mean, sum of squared differences)
    int C, HW, G, cg;         // channels, pixels, groups, channels per group
    int ldx, ldr, ldy, act;
    float eps;
    int gb, cb;               // groups and channels of a workgroup
    int upx, ug;              // units of V channels per pixel of a workgroup and per group
    int R, iters;             // pixels the threads cover at once, and how often (held)
    int n_cb;                 // workgroups side by side in the channels
    int chunks, chunk;        // two launches: chunks of an image and their pixels
    int total, per_die;       // workgroups, and a die's share of them
    FastDiv d_upx, d_ug, d_ncb, d_chunks;
};

template <int UB> struct RawUnit;
template <> struct RawUnit<2> { typedef unsigned short Type; };
template <> struct RawUnit<4> { typedef unsigned Type; };
template <> struct RawUnit<8> { typedef __attribute__((ext_vector_type(2))) unsigned Type; };
template <> struct RawUnit<16> { typedef __attribute__((ext_vector_type(4))) unsigned Type; };

typedef __amdgpu_buffer_rsrc_t Rsrc;
__device__ __forceinline__ Rsrc make_rsrc(const void *p, unsigned bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000);
}

template <int UB>
__device__ __forceinline__ typename RawUnit<UB>::Type load_unit(const Rsrc rs, unsigned off) {
    if constexpr (UB == 2) return __builtin_amdgcn_raw_buffer_load_b16(rs, off, 0, 0);
    else if constexpr (UB == 4) return __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, 0);
    else if constexpr (UB == 8) return __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
}
template <int UB>
__device__ __forceinline__ void store_unit(const Rsrc rs, unsigned off, typename RawUnit<UB>::Type v) {
    if constexpr (UB == 2) __builtin_amdgcn_raw_buffer_store_b16(v, rs, off, 0, 0);
    else if constexpr (UB == 4) __builtin_amdgcn_raw_buffer_store_b32(v, rs, off, 0, 0);
    else if constexpr (UB == 8) __builtin_amdgcn_raw_buffer_store_b64(v, rs, off, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(v, rs, off, 0, 0);
}

template <typename T, int V>
__device__ __forceinline__ void unpack(const typename RawUnit<V * sizeof(T)>::Type &u, float (&f)[V]) {
    T e[V];
    __builtin_memcpy(e, &u, sizeof(e));
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = static_cast<float>(e[i]);
}
template <typename T, int V>
__device__ __forceinline__ typename RawUnit<V * sizeof(T)>::Type pack(const float (&f)[V]) {
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = static_cast<T>(f[i]);
    typename RawUnit<V * sizeof(T)>::Type u;
    __builtin_memcpy(&u, e, sizeof(e));
    return u;
}

// Sum over a wavefront, the same in every lane: within rows of 16 lanes by DPP, then one lane of each row.
__device__ __forceinline__ float wave_sum(float v) {
    auto dpp = [](float f, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(f), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += dpp(v, std::integral_constant<int, 0xB1>());    // lane ^ 1
    v += dpp(v, std::integral_constant<int, 0x4E>());    // lane ^ 2
    v += dpp(v, std::integral_constant<int, 0x141>());   // mirrored within 8
    v += dpp(v, std::integral_constant<int, 0x140>());   // mirrored within 16
    const int i = __float_as_int(v);
    return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}

// Sum of `v` over the threads of the calling thread's group; threads of no unit pass zero.  `part`: one float per thread
// of LDS, `res`: kMaxGb floats, neither in use by anybody else.  The order of the sum depends on nothing but the geometry.
__device__ __forceinline__ float group_sum(float v, const Params &p, int my_group, float *part, float *res) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    if (p.gb == 1) {
        v = wave_sum(v);
        if (lane == 0) res[wave] = v;
        __syncthreads();
        float s = 0.f;
        for (int i = 0; i < waves; ++i) s += res[i];
        return s;
    }
    part[threadIdx.x] = v;
    __syncthreads();
    for (int g = wave; g < p.gb; g += waves) {
        float s = 0.f;
        for (int i = lane; i < p.R * p.ug; i += 64) {
            const int row = fdiv(i, p.d_ug);
            s += part[row * p.upx + g * p.ug + (i - row * p.ug)];
        }
        s = wave_sum(s);
        if (lane == 0) res[g] = s;
    }
    __syncthreads();
    return res[my_group];
}

// The unit of a thread: its row among the R pixels covered at once (or none), its channels and their scale and shift.
template <int V>
struct Place {
    int row, c, group;   // c: first channel, counted from the workgroup's first
    bool in;
    __device__ __forceinline__ Place(const Params &p) {
        row = fdiv(threadIdx.x, p.d_upx);
        const int u = threadIdx.x - row * p.upx;
        c = u * V;
        group = fdiv(u, p.d_ug);
        in = row < p.R;
    }
};

template <int V>
__device__ __forceinline__ void load_affine(const Params &p, int c, float (&a)[V], float (&b)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        a[i] = p.gamma ? p.gamma[c + i] : 1.f;
        b[i] = p.beta ? p.beta[c + i] : 0.f;
    }
}

// One unit from raw to stored form.
template <typename T, int V>
__device__ __forceinline__ typename RawUnit<V * sizeof(T)>::Type finish_unit(const typename RawUnit<V * sizeof(T)>::Type &x,
                                                                             const typename RawUnit<V * sizeof(T)>::Type &r, bool res,
                                                                             float mean, const float (&a)[V], const float (&b)[V],
                                                                             int act) {
    float f[V];
    unpack<T, V>(x, f);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (f[i] - mean) * a[i] + b[i];
    if (res) {
        float g[V];
        unpack<T, V>(r, g);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] += g[i];
    }
    activate(f, act);
    return pack<T, V>(f);
}

// Held: gb groups of one image in the registers of a workgroup, NR units a thread.
template <typename T, int V, int NR>
__global__ __launch_bounds__(kMaxThreads) void held_kernel(Params p) {
    constexpr int UB = V * static_cast<int>(sizeof(T));
    typedef typename RawUnit<UB>::Type Raw;
    constexpr bool EARLY_RES = NR * UB <= 64;   // the residual, too, is requested before the statistics
    __shared__ float part[kMaxThreads], res1[kMaxGb], res2[kMaxGb];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int n = fdiv(id, p.d_ncb), c0 = (id - n * p.n_cb) * p.cb;
    const Place<V> at(p);
    const size_t px = static_cast<size_t>(n) * p.HW;
    auto image = [&](const void *q, int ld) {
        return make_rsrc(static_cast<const char *>(q) + (px * ld + c0) * sizeof(T),
                         (static_cast<unsigned>(p.HW - 1) * ld + p.cb) * static_cast<unsigned>(sizeof(T)));
    };
    const Rsrc xs = image(p.x, p.ldx), ys = image(p.y, p.ldy), rs = p.r ? image(p.r, p.ldr) : xs;
    auto offset = [&](int i, int ld) {
        const int q = at.row + i * p.R;
        return at.in && q < p.HW ? static_cast<unsigned>(q * ld + at.c) * static_cast<unsigned>(sizeof(T)) : OOB;
    };
    Raw xv[NR], rv[EARLY_RES ? NR : 1];
#pragma unroll
    for (int i = 0; i < NR; ++i) xv[i] = load_unit<UB>(xs, offset(i, p.ldx));
    if (EARLY_RES && p.r) {
#pragma unroll
        for (int i = 0; i < (EARLY_RES ? NR : 1); ++i) rv[i] = load_unit<UB>(rs, offset(i, p.ldr));
    }
    float a[V], b[V];
    load_affine<V>(p, c0 + (at.in ? at.c : 0), a, b);
    const float inv = 1.f / (static_cast<float>(p.HW) * static_cast<float>(p.cg));
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        float f[V];
        unpack<T, V>(xv[i], f);
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) t += f[j];
        s += t;
    }
    const float mean = group_sum(s, p, at.group, part, res1) * inv;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        float f[V];
        unpack<T, V>(xv[i], f);
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) t += (f[j] - mean) * (f[j] - mean);
        s += at.in && at.row + i * p.R < p.HW ? t : 0.f;
    }
    const float var = group_sum(s, p, at.group, part, res2) * inv;
    const float rstd = 1.f / __builtin_sqrtf(var + p.eps);
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] *= rstd;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        Raw r{};
        if (p.r) r = EARLY_RES ? rv[EARLY_RES ? i : 0] : load_unit<UB>(rs, offset(i, p.ldr));
        store_unit<UB>(ys, offset(i, p.ldy), finish_unit<T, V>(xv[i], r, p.r != nullptr, mean, a, b, p.act));
    }
}

// Joins the statistics (count, mean, sum of squared differences) of two disjoint sets; an empty one counts for nothing.
struct Stat {
    float n, mean, m2;
};
__device__ __forceinline__ Stat join(const Stat a, const Stat b) {
    const float n = a.n + b.n;
    const float f = n > 0.f ? b.n / n : 0.f;
    const float d = b.mean - a.mean;
    return Stat{n, a.mean + d * f, a.m2 + b.m2 + d * d * a.n * f};
}
__device__ __forceinline__ Stat join_lanes(Stat s, int width) {
    for (int d = 1; d < width; d <<= 1) s = join(s, Stat{__shfl_xor(s.n, d), __shfl_xor(s.mean, d), __shfl_xor(s.m2, d)});
    return s;
}

constexpr int kBatch = 8;   // units in flight a thread

// Statistics of one chunk of an image for the groups of a workgroup.  A thread takes kBatch units at a time: their mean and
// squared differences from it, joined to what it has.
template <typename T, int V>
__global__ __launch_bounds__(kMaxThreads) void stats_kernel(Params p) {
    constexpr int UB = V * static_cast<int>(sizeof(T));
    typedef typename RawUnit<UB>::Type Raw;
    __shared__ float part[3][kMaxThreads];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int t = fdiv(id, p.d_ncb), cblk = id - t * p.n_cb, n = fdiv(t, p.d_chunks), k = t - n * p.chunks;
    const int c0 = cblk * p.cb, q0 = k * p.chunk, q1 = min(p.HW, q0 + p.chunk);
    const Place<V> at(p);
    const Rsrc xs = make_rsrc(static_cast<const char *>(p.x) + (static_cast<size_t>(n) * p.HW * p.ldx + c0) * sizeof(T),
                              (static_cast<unsigned>(p.HW - 1) * p.ldx + p.cb) * static_cast<unsigned>(sizeof(T)));
    Stat s{0.f, 0.f, 0.f};
    for (int q = q0 + at.row; q < q1 && at.in; q += kBatch * p.R) {
        Raw xv[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int qi = q + i * p.R;
            xv[i] = load_unit<UB>(xs, qi < q1 ? static_cast<unsigned>(qi * p.ldx + at.c) * static_cast<unsigned>(sizeof(T)) : OOB);
        }
        float sum = 0.f, cnt = 0.f;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            float f[V], u = 0.f;
            unpack<T, V>(xv[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) u += f[j];
            sum += u;
            cnt += q + i * p.R < q1 ? static_cast<float>(V) : 0.f;
        }
        const float mean = sum / cnt;
        float m2 = 0.f;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            float f[V], u = 0.f;
            unpack<T, V>(xv[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) u += (f[j] - mean) * (f[j] - mean);
            m2 += q + i * p.R < q1 ? u : 0.f;
        }
        s = join(s, Stat{cnt, mean, m2});
    }
    part[0][threadIdx.x] = s.n;
    part[1][threadIdx.x] = s.mean;
    part[2][threadIdx.x] = s.m2;
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    for (int g = wave; g < p.gb; g += waves) {
        Stat v{0.f, 0.f, 0.f};
        for (int i = lane; i < p.R * p.ug; i += 64) {
            const int row = fdiv(i, p.d_ug), j = row * p.upx + g * p.ug + (i - row * p.ug);
            v = join(v, Stat{part[0][j], part[1][j], part[2][j]});
        }
        v = join_lanes(v, 64);
        if (lane == 0) p.part[(static_cast<size_t>(n) * p.G + cblk * p.gb + g) * p.chunks + k] = make_float2(v.mean, v.m2);
    }
}

// Normalises one chunk of an image.
template <typename T, int V>
__global__ __launch_bounds__(kMaxThreads) void apply_kernel(Params p) {
    constexpr int UB = V * static_cast<int>(sizeof(T));
    typedef typename RawUnit<UB>::Type Raw;
    __shared__ float2 stat[kMaxGb];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int t = fdiv(id, p.d_ncb), cblk = id - t * p.n_cb, n = fdiv(t, p.d_chunks), k = t - n * p.chunks;
    const int c0 = cblk * p.cb, q0 = k * p.chunk, q1 = min(p.HW, q0 + p.chunk);
    const Place<V> at(p);
    const size_t px = static_cast<size_t>(n) * p.HW;
    auto image = [&](const void *q, int ld) {
        return make_rsrc(static_cast<const char *>(q) + (px * ld + c0) * sizeof(T),
                         (static_cast<unsigned>(p.HW - 1) * ld + p.cb) * static_cast<unsigned>(sizeof(T)));
    };
    const Rsrc xs = image(p.x, p.ldx), ys = image(p.y, p.ldy), rs = p.r ? image(p.r, p.ldr) : xs;
    float a[V], b[V];
    load_affine<V>(p, c0 + (at.in ? at.c : 0), a, b);
    // sixteen lanes join the chunks of a group
    for (int g = threadIdx.x >> 4; g < p.gb; g += blockDim.x >> 4) {
        const float2 *q = p.part + (static_cast<size_t>(n) * p.G + cblk * p.gb + g) * p.chunks;
        Stat v{0.f, 0.f, 0.f};
        for (int i = threadIdx.x & 15; i < p.chunks; i += 16) {
            const float2 e = q[i];
            v = join(v, Stat{static_cast<float>((min(p.HW, (i + 1) * p.chunk) - i * p.chunk)) * static_cast<float>(p.cg), e.x, e.y});
        }
        v = join_lanes(v, 16);
        if ((threadIdx.x & 15) == 0) stat[g] = make_float2(v.mean, 1.f / __builtin_sqrtf(v.m2 / v.n + p.eps));
    }
    __syncthreads();
    if (!at.in) return;
    const float mean = stat[at.group].x, rstd = stat[at.group].y;
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] *= rstd;
    for (int q = q0 + at.row; q < q1; q += kBatch * p.R) {
        Raw xv[kBatch], rv[kBatch];
        auto offset = [&](int i, int ld) {
            const int qi = q + i * p.R;
            return qi < q1 ? static_cast<unsigned>(qi * ld + at.c) * static_cast<unsigned>(sizeof(T)) : OOB;
        };
#pragma unroll
        for (int i = 0; i < kBatch; ++i) xv[i] = load_unit<UB>(xs, offset(i, p.ldx));
        if (p.r) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) rv[i] = load_unit<UB>(rs, offset(i, p.ldr));
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            store_unit<UB>(ys, offset(i, p.ldy), finish_unit<T, V>(xv[i], p.r ? rv[i] : xv[i], p.r != nullptr, mean, a, b, p.act));
    }
}

// One workgroup per image and group, element by element: groups of more than kMaxThreads units.
template <typename T>
__global__ __launch_bounds__(kMaxThreads) void wide_kernel(Params p) {
    __shared__ float res1[kMaxGb], res2[kMaxGb];
    const int n = fdiv(blockIdx.x, p.d_ncb), g = blockIdx.x - n * p.n_cb;
    const size_t px = static_cast<size_t>(n) * p.HW;
    const T *x = static_cast<const T *>(p.x) + px * p.ldx + g * p.cg;
    const T *r = p.r ? static_cast<const T *>(p.r) + px * p.ldr + g * p.cg : nullptr;
    T *y = static_cast<T *>(p.y) + px * p.ldy + g * p.cg;
    const float inv = 1.f / (static_cast<float>(p.HW) * static_cast<float>(p.cg));
    float mean = 0.f, rstd = 0.f;
    for (int pass = 0; pass < 3; ++pass) {
        float s = 0.f, t = 0.f;
        for (int q = 0; q < p.HW; ++q) {
            for (int c = threadIdx.x; c < p.cg; c += kMaxThreads) {
                float v[1] = {static_cast<float>(x[q * p.ldx + c])};
                if (pass == 0) {
                    t += v[0];
                } else if (pass == 1) {
                    t += (v[0] - mean) * (v[0] - mean);
                } else {
                    v[0] = (v[0] - mean) * (p.gamma ? rstd * p.gamma[g * p.cg + c] : rstd) + (p.beta ? p.beta[g * p.cg + c] : 0.f);
                    if (r) v[0] += static_cast<float>(r[q * p.ldr + c]);
                    activate(v, p.act);
                    y[q * p.ldy + c] = static_cast<T>(v[0]);
                }
            }
            if ((q & 255) == 255) {   // short partial sums: fewer roundings of a large one
                s += t;
                t = 0.f;
            }
        }
        s += t;
        if (pass == 0) mean = group_sum(s, p, 0, nullptr, res1) * inv;
        else if (pass == 1) rstd = 1.f / __builtin_sqrtf(group_sum(s, p, 0, nullptr, res2) * inv + p.eps);
    }
}

// ---- host side

constexpr size_t kHeldBytes = 96 << 10;   // of a group: see DESIGN
constexpr int kHeldDwords = 40;           // registers of a thread that hold units
constexpr size_t kChunkBytes = 128 << 10;
constexpr int kMaxChunks = 64;

struct Plan {
    enum Form { HELD, TWO, WIDE } form;
    int V, threads, iters;
    Params p;
};

void set_blocks(Plan &pl, int N, int per_image) {
    pl.p.total = N * per_image;
    pl.p.per_die = (pl.p.total + 7) / 8;
}

void set_units(Params &p, int V, int gb, int threads) {
    p.gb = gb;
    p.cb = gb * p.cg;
    p.upx = p.cb / V;
    p.ug = p.cg / V;
    p.R = threads / p.upx;
    p.n_cb = p.G / gb;
    p.d_upx = make_fastdiv(p.upx);
    p.d_ug = make_fastdiv(p.ug);
    p.d_ncb = make_fastdiv(p.n_cb);
}

Plan make_plan(const GroupNormArgs &a) {
    Plan pl{};
    Params &p = pl.p;
    p.x = a.x; p.r = a.residual; p.gamma = a.gamma; p.beta = a.beta; p.y = a.y;
    p.C = a.C; p.HW = a.H * a.W; p.G = a.groups; p.cg = a.C / a.groups;
    p.ldx = a.ldx; p.ldr = a.ldr; p.ldy = a.ldy;
    p.act = a.act; p.eps = a.eps;
    const int es = a.dtype == GPULET_F32 ? 4 : 2;
    int V = 16 / es;
    auto aligned = [&](const void *q, int ld) {
        return !q || (reinterpret_cast<uintptr_t>(q) % (V * es) == 0 && static_cast<size_t>(ld) % V == 0);
    };
    while (V > 1 && !(p.cg % V == 0 && aligned(a.x, a.ldx) && aligned(a.y, a.ldy) && aligned(a.residual, a.ldr))) V >>= 1;
    pl.V = V;
    p.chunks = 1;
    p.chunk = p.HW;
    p.d_chunks = make_fastdiv(1);
    if (p.cg / V > kMaxThreads) {
        pl.form = Plan::WIDE;
        set_units(p, p.cg, 1, 1);
        pl.threads = kMaxThreads;
        set_blocks(pl, a.N, p.G);
        return pl;
    }
    const int unit_dwords = std::max(1, V * es / 4);
    const size_t group_bytes = static_cast<size_t>(p.HW) * p.cg * es;
    // groups side by side until a pixel's piece is 64 bytes, half a line
    int gb = 1;
    while (gb < kMaxGb && gb < p.G && gb * p.cg * es < 64) {
        do ++gb; while (p.G % gb != 0);
    }
    if (gb > kMaxGb) gb = 1;
    if (group_bytes <= kHeldBytes) {
        for (int g = gb; g >= 1; --g) {
            if (p.G % g != 0 || g * p.cg / V > kMaxThreads) continue;
            // the fewest threads that hold the groups in two dwords' worth of 16-byte units each, or else as few as possible
            for (int threads = 64; threads <= kMaxThreads; threads *= 2) {
                const int upx = g * p.cg / V;
                if (upx > threads) continue;
                const int iters = (p.HW + threads / upx - 1) / (threads / upx);
                if (iters * unit_dwords > (threads < kMaxThreads ? 8 : kHeldDwords)) continue;
                pl.form = Plan::HELD;
                pl.threads = threads;
                pl.iters = iters;
                set_units(p, V, g, threads);
                set_blocks(pl, a.N, p.n_cb);
                return pl;
            }
        }
    }
    pl.form = Plan::TWO;
    // a pixel's piece of 256 bytes, or all of a group
    gb = 1;
    while (gb < p.G && gb * p.cg * es < 256) {
        int next = gb + 1;
        while (p.G % next != 0) ++next;
        if (next > kMaxGb || next * p.cg / V > kMaxThreads) break;
        gb = next;
    }
    pl.threads = std::max(256, (gb * p.cg / V + 63) / 64 * 64);
    set_units(p, V, gb, pl.threads);
    const size_t bytes = static_cast<size_t>(p.HW) * p.cb * es;
    const int chunks = static_cast<int>(std::min<size_t>(kMaxChunks, std::max<size_t>(1, bytes / kChunkBytes)));
    p.chunk = (p.HW + chunks - 1) / chunks;
    p.chunks = (p.HW + p.chunk - 1) / p.chunk;
    p.d_chunks = make_fastdiv(p.chunks);
    set_blocks(pl, a.N, p.n_cb * p.chunks);
    return pl;
}

template <typename T, int V>
hipError_t launch_units(const Plan &pl, hipStream_t stream) {
    const dim3 grid(8 * pl.p.per_die), block(pl.threads);
    constexpr int UD = V * sizeof(T) >= 4 ? V * sizeof(T) / 4 : 1;   // dwords of a unit
    if (pl.form == Plan::HELD) {
        if (pl.iters * UD <= 8) held_kernel<T, V, 8 / UD><<<grid, block, 0, stream>>>(pl.p);
        else if (pl.iters * UD <= 20) held_kernel<T, V, 20 / UD><<<grid, block, 0, stream>>>(pl.p);
        else held_kernel<T, V, kHeldDwords / UD><<<grid, block, 0, stream>>>(pl.p);
        return hipGetLastError();
    }
    stats_kernel<T, V><<<grid, block, 0, stream>>>(pl.p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    apply_kernel<T, V><<<grid, block, 0, stream>>>(pl.p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const Plan &pl, hipStream_t stream) {
    if (pl.form == Plan::WIDE) {
        wide_kernel<T><<<dim3(pl.p.total), kMaxThreads, 0, stream>>>(pl.p);
        return hipGetLastError();
    }
    switch (pl.V) {
        case 8:
            if constexpr (sizeof(T) == 2) return launch_units<T, 8>(pl, stream);
            return hipErrorInvalidValue;
        case 4: return launch_units<T, 4>(pl, stream);
        case 2: return launch_units<T, 2>(pl, stream);
        default: return launch_units<T, 1>(pl, stream);
    }
}

}  // namespace

hipError_t launch_group_norm(const GroupNormArgs &a, const LaunchCtx &ctx, hipStream_t stream) {
    Plan pl = make_plan(a);
    pl.p.part = static_cast<float2 *>(a.ws);
    if (a.dtype == GPULET_BF16) return launch_type<__bf16>(pl, stream);
    if (a.dtype == GPULET_F16) return launch_type<_Float16>(pl, stream);
    return launch_type<float>(pl, stream);
}

size_t group_norm_workspace(const GroupNormArgs &a) {
    const Plan pl = make_plan(a);
    return pl.form == Plan::TWO ? static_cast<size_t>(a.N) * a.groups * pl.p.chunks * sizeof(float2) : 0;
}

}  // namespace gpulet

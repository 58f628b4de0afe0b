// Group norm with residual and activation over NHWC maps (layers of the forward pass of a served network, paper Sec. 5):
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c] + r)
// with mean and var over the H x W x C / groups values of an image's group of channels.  Statistics are in fp32, the
// variance as the mean square of the differences from a mean (not of the values, which loses it where the mean is large).
//
// Bound by memory: x is read once and y written once, with about 14 vector operations an element.  Two forms:
//
// * held: a workgroup keeps whole groups of one image in registers: one launch, x read once.  For up to kHeldBytes.
// * two launches for larger groups: the first reduces chunks of an image to (mean, sum of squared differences) per group,
//   the second joins them and reads x again, from the last-level cache where x fits there.  8 maps of 256x256x128 (134 MB)
//   take 21 + 42 us, as much as 4.3 TB/s of the 268 MB that have to move; a copy of that size reaches 5.1.
//
// A single launch that holds what it read while all workgroups of an image exchange their sums would have to wait for
// workgroups that may not be running: another launch of the same kind on another stream could hold their places.
//
// Which one runs depends on the shape of an image and the alignment of its rows only, not on how many images there are or
// on the CUs of the gpu-let, so that an image's result has the same bits in any batch.
//
// A thread handles units of V consecutive channels of one group (V the largest power of two that divides the group and keeps
// all tensors' rows aligned, 16 bytes at most) and keeps its channels from pixel to pixel, so that its scale and shift stay
// in registers; the threads of a workgroup cover consecutive units of a pixel, then the next pixel.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

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
    int threads;              // of a workgroup
    int gb, cb;               // groups and channels of a workgroup
    int upx, ug;              // units of V channels per pixel of a workgroup and per group in it
    int slices, gu;           // two launches: workgroups that share the channels of a group (gb = 1), units of a whole group
    int R, iters;             // pixels the threads cover at once, and how often (held)
    int lanes;                // threads that join the values of a group: a power of two up to 64, all groups at once if it can
    int n_cb;                 // workgroups side by side in the channels
    int chunks, chunk;        // two launches: chunks of an image and their pixels
    int stat_chunks, stat_chunk;   // normalising launch: the same of the launch before
    int total, per_die;       // workgroups, and a die's share of them
    FastDiv d_upx, d_ug, d_ncb, d_chunks, d_slices;
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
__device__ __forceinline__ typename RawUnit<UB>::Type load_unit(const Rsrc rs, unsigned off, unsigned soff = 0) {
    if constexpr (UB == 2) return __builtin_amdgcn_raw_buffer_load_b16(rs, off, soff, 0);
    else if constexpr (UB == 4) return __builtin_amdgcn_raw_buffer_load_b32(rs, off, soff, 0);
    else if constexpr (UB == 8) return __builtin_amdgcn_raw_buffer_load_b64(rs, off, soff, 0);
    else return __builtin_amdgcn_raw_buffer_load_b128(rs, off, soff, 0);
}
// NT: not to be kept in the caches.  The scalar part of the offset is added to the vector part: a 16-byte buffer store with a
// scalar offset stored what the next vector instruction wrote to its first data register, in the last four of every 16
// lanes.  The compiler keeps the two apart only where the store has no scalar offset.
template <int UB, bool NT = false>
__device__ __forceinline__ void store_unit(const Rsrc rs, unsigned off, unsigned soff, typename RawUnit<UB>::Type v) {
    constexpr int AUX = NT ? 2 : 0;
    if constexpr (UB == 2) __builtin_amdgcn_raw_buffer_store_b16(v, rs, off + soff, 0, AUX);
    else if constexpr (UB == 4) __builtin_amdgcn_raw_buffer_store_b32(v, rs, off + soff, 0, AUX);
    else if constexpr (UB == 8) __builtin_amdgcn_raw_buffer_store_b64(v, rs, off + soff, 0, AUX);
    else __builtin_amdgcn_raw_buffer_store_b128(v, rs, off + soff, 0, AUX);
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

// The value of a lane of the other half among 2^(STEP + 1) lanes, once all lanes of each half agree (up to the order their
// values were joined in): within rows of 16 lanes by DPP.
template <int STEP>
__device__ __forceinline__ float other_half(float f) {
    if constexpr (STEP < 4) {
        constexpr int CTRL = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;   // lane ^ 1, lane ^ 2, mirrored within 8, 16
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(f), CTRL, 0xf, 0xf, true));
    } else {
        return __shfl_xor(f, 1 << STEP);
    }
}

// Sums over the first `lanes` (a power of two), the second, ... lanes of a wavefront.
template <int K, int STEP = 0>
__device__ __forceinline__ void lane_sums(float (&v)[K], int lanes) {
    if ((1 << STEP) >= lanes) return;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += other_half<STEP>(v[k]);
    if constexpr (STEP < 5) lane_sums<K, STEP + 1>(v, lanes);
}

// Replaces each of the K values by its sum over the threads of the calling thread's group; threads of no unit pass zero.
// `part`: K floats per thread of LDS, `res`: K per group or wavefront, neither in use by anybody else; `part` is free again on
// return.  The order of the sum depends on nothing but the geometry.
template <int K>
__device__ __forceinline__ void group_sums(float (&v)[K], const Params &p, int my_group, float (*part)[K], float (*res)[K]) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    if (p.gb == 1) {
        lane_sums(v, 16);   // within rows; the rows' sums go through scalar registers, which takes no trip to LDS
        auto row = [](float f, int r) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), 16 * r)); };
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = (row(v[k], 0) + row(v[k], 1)) + (row(v[k], 2) + row(v[k], 3));
        if (lane == 0) __builtin_memcpy(res[wave], v, sizeof(v));
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = 0.f;
        for (int i = 0; i < waves; ++i)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += res[i][k];
        return;
    }
    __builtin_memcpy(part[threadIdx.x], v, sizeof(v));
    __syncthreads();
    const int sub = threadIdx.x & (p.lanes - 1);
    for (int g = threadIdx.x / p.lanes; g < p.gb; g += blockDim.x / p.lanes) {
        float s[K] = {};
        for (int i = sub; i < p.R * p.ug; i += p.lanes) {
            const int row = fdiv(i, p.d_ug);
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] += part[row * p.upx + g * p.ug + (i - row * p.ug)][k];
        }
        lane_sums(s, p.lanes);
        if (sub == 0) __builtin_memcpy(res[g], s, sizeof(s));
    }
    __syncthreads();
    __builtin_memcpy(v, res[my_group], sizeof(v));
}

// The unit of a thread: its row among the R pixels covered at once (or none), its channels and their scale and shift.
template <int V>
struct Place {
    int row, c, group;   // c: first channel, counted from the workgroup's first
    bool in;
    __device__ __forceinline__ Place(const Params &p, int slice = 0) {
        row = fdiv(threadIdx.x, p.d_upx);
        const int u = threadIdx.x - row * p.upx;
        c = u * V;
        group = fdiv(u, p.d_ug);
        in = row < p.R && (p.slices == 1 || slice * p.upx + u < p.gu);
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
template <typename T, int V, ActCode A>
__device__ __forceinline__ typename RawUnit<V * sizeof(T)>::Type finish_unit(const typename RawUnit<V * sizeof(T)>::Type &x,
                                                                             const typename RawUnit<V * sizeof(T)>::Type &r, bool res,
                                                                             float mean, const float (&a)[V], const float (&b)[V],
                                                                             int act) {
    float f[V];
    unpack<T, V>(x, f);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (f[i] - mean) * a[i] + b[i];   // the shift minus mean * a would lose what is near the mean
    if (res) {
        float g[V];
        unpack<T, V>(r, g);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] += g[i];
    }
    activate<A>(f, act);
    return pack<T, V>(f);
}

// Held: gb groups of one image in the registers of a workgroup, NR units a thread.  Two units of 8 channels take 66 registers
// if they may; with 64 a second workgroup of 1024 threads has room on a CU (32 images of 16x16x1280 22 us instead of 28).
template <typename T, int V, int NR, ActCode A>
__global__ __launch_bounds__(kMaxThreads, V == 8 && NR == 2 ? 8 : 4) void held_kernel(Params p) {
    constexpr int UB = V * static_cast<int>(sizeof(T));
    typedef typename RawUnit<UB>::Type Raw;
    constexpr bool EARLY_RES = NR * UB <= 64;   // the residual, too, is requested before the statistics
    extern __shared__ float2 part[];   // one per thread where the workgroup has several groups (held_lds), for both sums
    __shared__ float res1[kMaxGb][1];
    __shared__ __attribute__((aligned(8))) float res2[kMaxGb][2];
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
    // Rows of pixels before row `full` are whole: their offset is the thread's own plus a scalar; row `full` may be short.
    const int full = p.iters - 1;
    const bool tail = at.in && at.row + full * p.R < p.HW;
    auto valid = [&](int i) { return i < full ? at.in : i == full && tail; };
    auto base = [&](int ld) { return static_cast<unsigned>(at.row * ld + at.c) * static_cast<unsigned>(sizeof(T)); };
    auto step = [&](int i, int ld) { return static_cast<unsigned>(min(i, full) * p.R * ld) * static_cast<unsigned>(sizeof(T)); };
    // For every register with a unit.  Where a thread has many, those without one are left out four at a time (7 images of
    // 11 x 18 x 96 in 32 groups, 10 units of 24: 7.3 us, computed for nothing 11.9); a test in front of few costs 3 %.
    auto units = [&](auto &&f) {
#pragma unroll
        for (int i0 = 0; i0 < NR; i0 += 4) {
            if (NR > 8 && i0 > full) continue;
#pragma unroll
            for (int i = i0; i < (i0 + 4 < NR ? i0 + 4 : NR); ++i) f(i);
        }
    };
    Raw xv[NR], rv[EARLY_RES ? NR : 1];
    const unsigned xo = base(p.ldx), yo = base(p.ldy), ro = base(p.ldr);
    units([&](int i) { xv[i] = load_unit<UB>(xs, valid(i) ? xo : OOB, step(i, p.ldx)); });
    if constexpr (EARLY_RES) {
        if (p.r) units([&](int i) { rv[i] = load_unit<UB>(rs, valid(i) ? ro : OOB, step(i, p.ldr)); });
    }
    // Of a group of equal values the mean is that value, to the bit: sums are of differences from its first value.  That one
    // may lie so far off that the roundings of such a sum count (16x16x32 fp32, one value far off: 4.5e-6 of a standard
    // deviation).  So it only gives `near`, the mean of some of the group's values, and the differences from that give what
    // is missing to the mean.  One value in twelve, at least, is enough: their mean is at most sqrt(11) standard deviations
    // away from that of all, where the squares' sum, with its 30 roundings, is twelve times the variance's.
    float first[1];
    unpack<T, 1>(load_unit<sizeof(T)>(xs, static_cast<unsigned>(at.group * p.cg) * static_cast<unsigned>(sizeof(T))), first);
    float a[V], b[V];
    load_affine<V>(p, c0 + (at.in ? at.c : 0), a, b);
    constexpr int SUB = (NR + 3) / 4, SV = V < 2 ? V : 2;   // units and values of each
    float s[1] = {};
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
        float f[V];
        unpack<T, V>(xv[i], f);
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < SV; ++j) t += f[j] - first[0];
        s[0] += valid(i) ? t : 0.f;
    }
    group_sums(s, p, at.group, reinterpret_cast<float(*)[1]>(part), res1);
    const float near = first[0] + s[0] * __builtin_amdgcn_rcpf(static_cast<float>(min(p.HW, SUB * p.R)) * static_cast<float>(p.gu * SV));
    const float inv = __builtin_amdgcn_rcpf(static_cast<float>(p.HW) * static_cast<float>(p.cg));
    float d[2] = {};
    units([&](int i) {
        float f[V];
        unpack<T, V>(xv[i], f);
        const float from = valid(i) ? near : 0.f;   // units left out were loaded as zeros
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float e = f[j] - from;
            d[0] += e;
            d[1] += e * e;
        }
    });
    group_sums(d, p, at.group, reinterpret_cast<float(*)[2]>(part), res2);
    const float more = d[0] * inv, mean = near + more;
    const float var = d[1] < __builtin_inff() ? fmaxf(d[1] * inv - more * more, 0.f) : d[1];
    const float rstd = 1.f / __builtin_sqrtf(var + p.eps);
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] *= rstd;
    units([&](int i) {
        Raw r{};
        if (p.r) r = EARLY_RES ? rv[EARLY_RES ? i : 0] : load_unit<UB>(rs, valid(i) ? ro : OOB, step(i, p.ldr));
        store_unit<UB>(ys, valid(i) ? yo : OOB, step(i, p.ldy), finish_unit<T, V, A>(xv[i], r, p.r != nullptr, mean, a, b, p.act));
    });
}

// Joins the statistics (count, mean, sum of squared differences) of two disjoint sets; an empty one, whose mean is zero,
// counts for nothing.  d * d alone may be more than fp32 holds where one set is empty and the other's mean is large.
struct Stat {
    float n, mean, m2;
};
// `d`: how far b's mean is from a's.
__device__ __forceinline__ Stat join(const Stat a, const Stat b, float d) {
    const float n = a.n + b.n;
    const float f = a.n > 0.f ? b.n * __builtin_amdgcn_rcpf(n) : 1.f;   // equal means stay what they are, to the bit
    return Stat{n, a.mean + d * f, a.m2 + b.m2 + d * (a.n * f) * d};
}
__device__ __forceinline__ Stat join(const Stat a, const Stat b) { return join(a, b, b.mean - a.mean); }
template <int STEP = 0>
__device__ __forceinline__ Stat join_lanes(Stat s, int lanes) {
    if ((1 << STEP) >= lanes) return s;
    s = join(s, Stat{other_half<STEP>(s.n), other_half<STEP>(s.mean), other_half<STEP>(s.m2)});
    if constexpr (STEP < 5) return join_lanes<STEP + 1>(s, lanes);
    return s;
}

// Units in flight a thread in the two launches.  Twice as many are no faster (5 images of 37 x 29 x 246 fp32 10.2 us instead
// of 9.2) and make longer code.
constexpr int batch_of(int unit_bytes) { return unit_bytes >= 8 ? 4 : 8; }

// A thread's walk over the pixels of a chunk, batch_of(UB) units at a time: `full` batches without a test, then one with.
// Steps to pixels behind the chunk may be longer than the image, so nothing is added to the offset of a unit that is left
// out: OOB and such a step in one sum may come out inside the image, and a scalar offset has to stay below the buffer's size.
template <typename T, int V>
struct Walk {
    static constexpr int UB = V * static_cast<int>(sizeof(T)), B = batch_of(UB);
    typedef typename RawUnit<UB>::Type Raw;
    int q, left;   // first pixel of the thread, pixels of the chunk from the first row on
    const Place<V> &at;
    const Params &p;
    __device__ __forceinline__ Walk(const Params &p_, const Place<V> &at_, int q0, int q1) : q(q0 + at_.row), left(q1 - q0), at(at_), p(p_) {}
    __device__ __forceinline__ bool full() const { return left >= B * p.R; }
    __device__ __forceinline__ bool valid(int i) const { return at.in && at.row + i * p.R < left; }
    __device__ __forceinline__ unsigned base(int ld) const {
        return at.in ? static_cast<unsigned>(q * ld + at.c) * static_cast<unsigned>(sizeof(T)) : OOB;
    }
    __device__ __forceinline__ unsigned step(int ld) const { return static_cast<unsigned>(p.R * ld) * static_cast<unsigned>(sizeof(T)); }
    __device__ __forceinline__ void load(const Rsrc rs, int ld, Raw (&v)[B]) const {
        const unsigned o = base(ld), d = step(ld);
        if (full()) {
#pragma unroll
            for (int i = 0; i < B; ++i) v[i] = load_unit<UB>(rs, o, i * d);
        } else {
#pragma unroll
            for (int i = 0; i < B; ++i) v[i] = load_unit<UB>(rs, valid(i) ? o : OOB, i * p.R < left ? i * d : 0u);
        }
    }
    // Vector offset of unit i for a store, `whole` where its batch is full and the thread has a unit.
    __device__ __forceinline__ unsigned store_at(int i, bool whole, unsigned o, unsigned d) const {
        return whole || valid(i) ? o + i * d : OOB;
    }
    __device__ __forceinline__ void next() {
        q += B * p.R;
        left -= B * p.R;
    }
};

// Statistics of one chunk of an image for the groups of a workgroup.  A thread sums the differences of a batch from the mean
// of what it summed before, and their squares, and joins the batch's statistics to those before; the first batch's are
// from the mean of a quarter of its values, at least.  The roundings of the squares' sum are at most B V 2^-24 of it.  Of the
// n0 + nb values joined so far, the nb new ones, whose mean is D away, add n0 nb / (n0 + nb) D^2, at least half of what their
// squares' sum has from D; the first batch's sum is at most four times what it is from the batch's own mean.  So the roundings
// are no more than 4 B V 2^-24 (8e-6) of the result, wherever the values lie.
// (One sum of differences from the thread's first value: up to 1e-2 of it where that value is the only one that lies far off.)
template <typename T, int V>
__global__ __launch_bounds__(kMaxThreads) void stats_kernel(Params p) {
    typedef Walk<T, V> W;
    __shared__ float part[3][kMaxThreads];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int t = fdiv(id, p.d_ncb), cblk = id - t * p.n_cb, n = fdiv(t, p.d_chunks), k = t - n * p.chunks;
    const int gblk = fdiv(cblk, p.d_slices), slice = cblk - gblk * p.slices, sc = slice * p.upx * V;
    const int c0 = gblk * p.cb + sc, q0 = k * p.chunk, q1 = min(p.HW, q0 + p.chunk);
    const Place<V> at(p, slice);
    const Rsrc xs = make_rsrc(static_cast<const char *>(p.x) + (static_cast<size_t>(n) * p.HW * p.ldx + c0) * sizeof(T),
                              (static_cast<unsigned>(p.HW - 1) * p.ldx + p.cb - sc) * static_cast<unsigned>(sizeof(T)));
    W w(p, at, q0, q1);
    typename W::Raw xv[W::B];
    w.load(xs, p.ldx, xv);
    // Calls f with the first N values of every unit of a batch, or with `none` for one that is not there.  -> how many are there
    auto each = [&](const typename W::Raw (&raw)[W::B], bool whole, float none, auto N, auto &&f) {
        int units = whole && at.in ? W::B : 0;
#pragma unroll
        for (int i = 0; i < W::B; ++i) {
            const bool ok = whole || w.valid(i);
            if (!whole) units += ok;
            float v[V];
            unpack<T, V>(raw[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) f(ok ? v[j] : none);
        }
        return static_cast<float>(units * N);
    };
    constexpr std::integral_constant<int, V> ALL{};
    constexpr std::integral_constant<int, V < 2 ? V : 2> SOME{};
    float first[V];
    unpack<T, V>(xv[0], first);
    float sum = 0.f;
    float nb = each(xv, w.full(), first[0], SOME, [&](float v) { sum += v - first[0]; });
    // of equal values the mean is that value, to the bit; of none it is zero
    Stat all{0.f, first[0] + sum * __builtin_amdgcn_rcpf(fmaxf(nb, 1.f)), 0.f};
    while (true) {
        typename W::Raw cur[W::B];
#pragma unroll
        for (int i = 0; i < W::B; ++i) cur[i] = xv[i];
        W next = w;
        next.next();
        const bool more = next.left > 0;
        if (more) next.load(xs, p.ldx, xv);   // on its way while the batch before is summed
        float sq = 0.f;
        sum = 0.f;
        nb = each(cur, w.full(), all.mean, ALL, [&](float v) {
            const float d = v - all.mean;
            sum += d;
            sq += d * d;
        });
        const float d = sum * __builtin_amdgcn_rcpf(fmaxf(nb, 1.f));
        // not below zero; where the squares overflow, infinite, as their sum is in the other form (not infinity less infinity)
        const float m2 = sq < __builtin_inff() ? fmaxf(sq - sum * d, 0.f) : sq;
        all = join(all, Stat{nb, all.mean + d, m2}, d);
        w.q = next.q;
        w.left = next.left;
        if (!more) break;
    }
    part[0][threadIdx.x] = all.n;
    part[1][threadIdx.x] = all.mean;
    part[2][threadIdx.x] = all.m2;
    __syncthreads();
    const int sub = threadIdx.x & (p.lanes - 1);
    for (int g = threadIdx.x / p.lanes; g < p.gb; g += blockDim.x / p.lanes) {
        Stat v{0.f, 0.f, 0.f};
        for (int i = sub; i < p.R * p.ug; i += p.lanes) {
            const int row = fdiv(i, p.d_ug), j = row * p.upx + g * p.ug + (i - row * p.ug);
            v = join(v, Stat{part[0][j], part[1][j], part[2][j]});
        }
        v = join_lanes(v, p.lanes);
        if (sub == 0) p.part[((static_cast<size_t>(n) * p.G + gblk * p.gb + g) * p.chunks + k) * p.slices + slice] = make_float2(v.mean, v.m2);
    }
}

// Normalises one chunk of an image.
template <typename T, int V, bool NT, ActCode A>
__global__ __launch_bounds__(kMaxThreads) void apply_kernel(Params p) {
    typedef Walk<T, V> W;
    __shared__ float2 stat[kMaxGb];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int t = fdiv(id, p.d_ncb), cblk = id - t * p.n_cb, n = fdiv(t, p.d_chunks), k = t - n * p.chunks;
    const int gblk = fdiv(cblk, p.d_slices), slice = cblk - gblk * p.slices, sc = slice * p.upx * V;
    const int c0 = gblk * p.cb + sc, q0 = k * p.chunk, q1 = min(p.HW, q0 + p.chunk);
    const Place<V> at(p, slice);
    const size_t px = static_cast<size_t>(n) * p.HW;
    auto image = [&](const void *q, int ld) {
        return make_rsrc(static_cast<const char *>(q) + (px * ld + c0) * sizeof(T),
                         (static_cast<unsigned>(p.HW - 1) * ld + p.cb - sc) * static_cast<unsigned>(sizeof(T)));
    };
    const Rsrc xs = image(p.x, p.ldx), ys = image(p.y, p.ldy), rs = p.r ? image(p.r, p.ldr) : xs;
    W w(p, at, q0, q1);
    typename W::Raw xv[W::B], rv[W::B];
    w.load(xs, p.ldx, xv);
    if (p.r) w.load(rs, p.ldr, rv);
    float a[V], b[V];
    load_affine<V>(p, c0 + (at.in ? at.c : 0), a, b);
    const int sub = threadIdx.x & (p.lanes - 1);
    for (int g = threadIdx.x / p.lanes; g < p.gb; g += blockDim.x / p.lanes) {
        const int parts = p.stat_chunks * p.slices;
        const float2 *q = p.part + (static_cast<size_t>(n) * p.G + gblk * p.gb + g) * parts;
        Stat v{0.f, 0.f, 0.f};
        for (int i = sub; i < parts; i += p.lanes) {
            const float2 e = q[i];
            const int chunk = fdiv(i, p.d_slices), first = chunk * p.stat_chunk;
            const int units = p.slices == 1 ? p.gu : min(p.upx, p.gu - (i - chunk * p.slices) * p.upx);
            v = join(v, Stat{static_cast<float>(min(p.HW - first, p.stat_chunk)) * static_cast<float>(units * V), e.x, e.y});
        }
        v = join_lanes(v, p.lanes);
        if (sub == 0) stat[g] = make_float2(v.mean, 1.f / __builtin_sqrtf(v.m2 / v.n + p.eps));
    }
    __syncthreads();
    const float mean = stat[at.group].x, rstd = stat[at.group].y;
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] *= rstd;
    while (true) {
        const unsigned o = w.base(p.ldy), d = w.step(p.ldy);
        const bool whole = w.full() && at.in;
#pragma unroll
        for (int i = 0; i < W::B; ++i) {
            const typename W::Raw y = finish_unit<T, V, A>(xv[i], p.r ? rv[i] : xv[i], p.r != nullptr, mean, a, b, p.act);
            store_unit<W::UB, NT>(ys, w.store_at(i, whole, o, d), 0u, y);
        }
        w.next();
        if (w.left <= 0) break;
        w.load(xs, p.ldx, xv);
        if (p.r) w.load(rs, p.ldr, rv);
    }
}

// ---- host side

// Bytes of the groups a workgroup holds, at most.  Above, too few workgroups read pieces of pixels too short for the memory
// system: held and in two launches took, bf16, 32 groups, in a graph,
//    5 KB  8x8x1280   1 image  4.3 and 7.7 us    32 images  7.7 and 10.6
//   12 KB  14x14x1024 1 image  4.6 and 7.4       32 images 10.6 and 14.6
//   20 KB  16x16x1280 1 image  7.6 and 7.7       32 images 21.8 and 20.7
//   49 KB  28x28x256  1 image 10.4 and 7.5       32 images 13.1 and 14.4
//   80 KB  32x32x1280 1 image 11.5 and 8.2       32 images 51.6 and 54.4
constexpr size_t kHeldBytes = 32 << 10;
constexpr int kHeldDwords = 24;           // registers of a thread that hold units
// Bytes of a workgroup's chunk.  Statistics: 32 chunks (one for each lane that joins them), unless they are out of these
// limits.  Normalising: an image is spread over 256 workgroups within these limits.
constexpr size_t kMinStats = 8 << 10, kMaxStats = 256 << 10, kMinApply = 8 << 10, kMaxApply = 32 << 10;
// Results of this size and more are stored past the caches: they would push out the x that is still to be read a second
// time, and most of them would be gone from the caches before anybody reads them.
constexpr size_t kStreamBytes = 64 << 20;

struct Plan {
    enum Form { HELD, TWO } form;
    int V, iters;
    bool stream_out, fits;
    Params p, q;   // of the only or first launch, and of the second
};

// -> whether a launch may have as many threads: fewer than 2^32.
bool set_blocks(Params &p, int N, long long per_image) {
    const long long total = N * per_image, per_die = (total + 7) / 8;
    if (8 * per_die * p.threads >= (1LL << 32)) return false;
    p.total = static_cast<int>(total);
    p.per_die = static_cast<int>(per_die);
    return true;
}

void set_units(Params &p, int V, int gb, int slices, int threads) {
    p.threads = threads;
    p.gb = gb;
    p.cb = gb * p.cg;
    p.slices = slices;
    p.gu = p.cg / V;
    p.ug = (p.gu + slices - 1) / slices;
    p.upx = gb * p.ug;
    p.R = threads / p.upx;
    p.lanes = 64;
    while (p.lanes > 1 && p.lanes * gb > threads) p.lanes /= 2;
    p.n_cb = p.G / gb * slices;
    p.d_slices = make_fastdiv(slices);
    p.d_upx = make_fastdiv(p.upx);
    p.d_ug = make_fastdiv(p.ug);
    p.d_ncb = make_fastdiv(p.n_cb);
}

// Chunks of about `piece` bytes, made of whole batches.
bool set_chunks(Params &p, int V, int unit_bytes, int gb, int slices, int threads, size_t block_bytes, size_t piece, int N) {
    set_units(p, V, gb, slices, threads);
    const int chunks = static_cast<int>(std::max<size_t>(1, block_bytes / piece));
    const int whole = p.R * batch_of(unit_bytes);
    p.chunk = ((p.HW + chunks - 1) / chunks + whole - 1) / whole * whole;
    p.chunks = (p.HW + p.chunk - 1) / p.chunk;
    p.d_chunks = make_fastdiv(p.chunks);
    return set_blocks(p, N, 1LL * p.n_cb * p.chunks);
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
    const int unit_dwords = std::max(1, V * es / 4);
    const size_t group_bytes = static_cast<size_t>(p.HW) * p.cg * es;
    // groups side by side until a pixel's piece is 64 bytes, half a line
    int gb = 1;
    while (gb < kMaxGb && gb < p.G && gb * p.cg * es < 64) {
        do ++gb; while (p.G % gb != 0);
    }
    if (gb > kMaxGb) gb = 1;
    if (group_bytes * gb <= kHeldBytes && gb * p.cg / V <= kMaxThreads) {
        // the fewest threads that hold the groups in 8 dwords each, or else as few dwords as possible
        const int upx = gb * p.cg / V;
        for (int threads = 64; threads <= kMaxThreads; threads *= 2) {
            if (upx > threads) continue;
            const int rows = threads / upx, iters = (p.HW + rows - 1) / rows;
            if (iters * unit_dwords > (threads < kMaxThreads ? 8 : kHeldDwords)) continue;
            pl.form = Plan::HELD;
            pl.iters = p.iters = iters;
            set_units(p, V, gb, 1, threads);
            pl.fits = set_blocks(p, a.N, p.n_cb);
            return pl;
        }
    }
    pl.form = Plan::TWO;
    // a pixel's piece of 128 bytes, a line, or all of a group
    gb = 1;
    while (gb < p.G && gb * p.cg * es < 128) {
        int next = gb + 1;
        while (p.G % next != 0) ++next;
        if (next > kMaxGb || next * p.cg / V > kMaxThreads) break;
        gb = next;
    }
    // a group of more units than a workgroup has threads is shared by several
    const int slices = (p.cg / V + kMaxThreads - 1) / kMaxThreads;
    const size_t block_bytes = static_cast<size_t>(p.HW) * gb * p.cg * es / slices;
    const size_t stats = std::min(kMaxStats, std::max(kMinStats, block_bytes / 32));
    const size_t apply = std::min(kMaxApply, std::max(kMinApply, block_bytes * slices * (p.G / gb) / 256));
    pl.stream_out = static_cast<size_t>(a.N) * p.HW * p.C * es >= kStreamBytes;
    pl.q = p;
    const int fewest = ((gb * p.cg / V + slices - 1) / slices + 63) / 64 * 64;   // threads of one row
    pl.fits = set_chunks(p, V, V * es, gb, slices, std::max(stats >= (64 << 10) ? 512 : 256, fewest), block_bytes, stats, a.N);
    pl.fits = set_chunks(pl.q, V, V * es, gb, slices, std::max(256, fewest), block_bytes, apply, a.N) && pl.fits;
    pl.q.stat_chunks = p.chunks;
    pl.q.stat_chunk = p.chunk;
    return pl;
}

// LDS of a held kernel's sums per thread: as many workgroups of 64 threads as a CU takes have room.
size_t held_lds(const Params &p) { return p.gb > 1 ? p.threads * sizeof(float2) : 0; }

template <typename T, int V, ActCode A>
hipError_t launch_units(const Plan &pl, hipStream_t stream) {
    const dim3 grid(8 * pl.p.per_die), block(pl.p.threads);
    constexpr int UD = V * sizeof(T) >= 4 ? V * sizeof(T) / 4 : 1;   // dwords of a unit
    if (pl.form == Plan::HELD) {
        const size_t lds = held_lds(pl.p);
        if (pl.iters * UD <= 8) held_kernel<T, V, 8 / UD, A><<<grid, block, lds, stream>>>(pl.p);
        else held_kernel<T, V, kHeldDwords / UD, A><<<grid, block, lds, stream>>>(pl.p);
        return hipGetLastError();
    }
    stats_kernel<T, V><<<grid, block, 0, stream>>>(pl.p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid2(8 * pl.q.per_die), block2(pl.q.threads);
    if (pl.stream_out) apply_kernel<T, V, true, A><<<grid2, block2, 0, stream>>>(pl.q);
    else apply_kernel<T, V, false, A><<<grid2, block2, 0, stream>>>(pl.q);
    return hipGetLastError();
}

template <typename T, ActCode A>
hipError_t launch_type(const Plan &pl, hipStream_t stream) {
    switch (pl.V) {
        case 8:
            if constexpr (sizeof(T) == 2) return launch_units<T, 8, A>(pl, stream);
            return hipErrorInvalidValue;
        case 4: return launch_units<T, 4, A>(pl, stream);
        case 2: return launch_units<T, 2, A>(pl, stream);
        default: return launch_units<T, 1, A>(pl, stream);
    }
}

template <typename T>
hipError_t launch_act(const Plan &pl, hipStream_t stream) {
    if (pl.p.act == GPULET_ACT_SILU) return launch_type<T, ActCode::SILU>(pl, stream);
    switch (act_code(pl.p.act)) {
        case ActCode::NORMAL: return launch_type<T, ActCode::NORMAL>(pl, stream);
        case ActCode::GATE: return launch_type<T, ActCode::GATE>(pl, stream);
        default: return launch_type<T, ActCode::LINEAR>(pl, stream);
    }
}

}  // namespace

hipError_t launch_group_norm(const GroupNormArgs &a, hipStream_t stream, int *launches) {
    Plan pl = make_plan(a);
    if (launches) *launches = pl.form == Plan::TWO ? 2 : 1;
    pl.p.part = pl.q.part = static_cast<float2 *>(a.ws);
    if (a.dtype == GPULET_BF16) return launch_act<__bf16>(pl, stream);
    if (a.dtype == GPULET_F16) return launch_act<_Float16>(pl, stream);
    return launch_act<float>(pl, stream);
}

bool group_norm_fits(const GroupNormArgs &a) { return make_plan(a).fits; }

size_t group_norm_workspace(const GroupNormArgs &a) {
    const Plan pl = make_plan(a);
    return pl.form == Plan::TWO ? static_cast<size_t>(a.N) * a.groups * pl.p.chunks * pl.p.slices * sizeof(float2) : 0;
}

}  // namespace gpulet

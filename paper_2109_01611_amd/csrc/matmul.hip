// Matrix product with bias, residual and activation in its epilogue on gfx950 matrix cores:
//   y[m, n] = act(sum_k x[m, k] w[n, k] + b[n] + r[m, n])
// for the per-pixel and per-row layers of a forward pass (paper Sec. 5) that a ReLU convolution or the fully connected
// layer cannot stand for: wide activations, fp16, fp32 results, rows that are slices of wider ones, any number of rows.
//
// Forms, chosen per call by an estimate of their times (choose_matmul).  Times are those of a call in a graph of 20.
//   ring     up to 64x64 of y a workgroup, whose wavefronts share the depth, each with slices of its own in LDS and no barrier
//            before the end.  Few rows, few tiles.  Bound by memory: 1 x 4096 x 4096 5.3 us (6.3 TB/s of the weights, part of
//            which are in the last-level cache), 24 x 1024 x 4096 4.7, 197 x 1024 x 4096 7.9.
//   tile     64x64, 128x64 and 128x128 tiles that a workgroup goes through slice by slice.  Bound by the rate at which a CU
//            takes operands (60 to 85 KB/us, whatever lies in flight): 6272 x 1024 x 4096 in 128x128 58 to 64 us, 820 to
//            900 TFLOP/s.
//            The 64x64 one also with a depth that up to eight workgroups share, whose sums meet in the workspace: tall y with
//            few tiles and a long depth (1742 x 216 x 3816 15.0 us, in rings 19.2).
//   big      256x256 tiles, 160 KB of LDS: as many matrix instructions as transfers can feed.  8192 x 4096 x 4096 216 us,
//            1.27 PFLOP/s (1.25 for the library's product of that size); 8192^3 820 us, 1.34.
//   direct,  rows that do not start at multiples of 16 bytes or a depth that is not a multiple of 8: operands go from memory
//   staged   into the matrix instructions (few rows, few tiles), or through registers into LDS (64x64 tiles).
//            200 x 300 x 4001 8.5 us.  Larger products of such operands lay them out anew in the workspace first and
//            take the forms above: 2048 x 1024 x 1001 18.2 us (staged 21.6), 4096 x 4096 x 1022 45 (84).
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
typedef __attribute__((ext_vector_type(4))) int i32x4;

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
    int tiles_m, tiles_n;
    int total, per_die;     // workgroups, and a die's share of them
    int splits;             // workgroups that share a tile
    int slices;             // slices of the depth: of 64, a workgroup's (splits > 1) or a wavefront's (ring); of 32, a
                            // wavefront's (direct)
    float *part;            // splits > 1: [split][M][N] sums
    int past;               // y goes past the caches
    FastDiv d_tiles, d_tiles_n, d_tiles_m;
};

// What the epilogue adds to NC consecutive columns of row m, asked for before it is needed: a workgroup with a short depth
// lives about as long as these loads take.  Rows of y and the residual may start anywhere: 16 bytes at a time they cost less
// than element by element at any alignment (12965 x 3053 x 280 bf16 153 us element by element, 65 so).
template <int NC>
__device__ __forceinline__ void load_bias(const Params &p, int n, float (&b)[NC]) {
#pragma unroll
    for (int i = 0; i < NC; ++i) b[i] = 0.f;
    if (!p.b) return;
    if (n + NC <= p.N) {
        __builtin_memcpy(b, p.b + n, sizeof(b));
        return;
    }
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (n + i < p.N) b[i] = p.b[n + i];
}
template <int NC, typename T>
__device__ __forceinline__ void load_residual(const Params &p, int m, int n, T (&r)[NC]) {
    if (!p.r || m >= p.M) return;
    const T *at = static_cast<const T *>(p.r) + static_cast<long long>(m) * p.ldr + n;
    if (n + NC <= p.N) {
        __builtin_memcpy(r, at, sizeof(r));
        return;
    }
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (n + i < p.N) r[i] = at[i];
}
// Bias, residual and activation, then the store.
template <int NC, typename T, ActCode A>
__device__ __forceinline__ void finish(const Params &p, int m, int n, const float (&bias)[NC], const T (&r)[NC], float (&v)[NC]) {
    T *y = static_cast<T *>(p.y) + static_cast<long long>(m) * p.ldy + n;
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] += bias[i];
    if (p.r) {
#pragma unroll
        for (int i = 0; i < NC; ++i) v[i] += static_cast<float>(r[i]);
    }
    activate<A>(v, p.act);
    T e[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) e[i] = static_cast<T>(v[i]);
    if (n + NC <= p.N) {
        if constexpr (sizeof(e) == 16) {
            if (p.past) {
                i32x4 q;
                __builtin_memcpy(&q, e, sizeof(e));
                __builtin_nontemporal_store(q, reinterpret_cast<i32x4 *>(y));
                return;
            }
        }
        __builtin_memcpy(y, e, sizeof(e));
        return;
    }
#pragma unroll
    for (int i = 0; i < NC; ++i)
        if (n + i < p.N) y[i] = e[i];
}

// The columns a lane of a tile kernel holds: run u is the 16 bytes of y from column u * 64 / sizeof(TO) + (lane / 16) *
// RUN on, so that a store of one run by a wavefront is 64 consecutive bytes in each of 16 rows.  (One run of 4 NB columns a
// lane leaves every second 16 bytes to the next store: 4096 x 4096 x 1024 41.9 us instead of 38.7.)
template <typename TO> constexpr int RUN = 16 / sizeof(TO);
// Stored row `in` of a wavefront's columns -> column.
template <typename TO>
__device__ __forceinline__ int column_of(int in) {
    constexpr int BLOCKS = RUN<TO> / 4;   // blocks of 16 rows to a run
    const int blk = in >> 4, s = in & 15;
    return blk / BLOCKS * 4 * RUN<TO> + (s >> 2) * RUN<TO> + blk % BLOCKS * 4 + (s & 3);
}
template <typename TO, int RUNS>
__device__ __forceinline__ void load_biases(const Params &p, int n, float (&b)[RUNS][RUN<TO>]) {
#pragma unroll
    for (int u = 0; u < RUNS; ++u) load_bias(p, n + u * 4 * RUN<TO>, b[u]);
}
// Rows m, m + 16, ... of a lane's accumulators from column n on; the residuals of G rows are asked for at a time.
template <typename TO, ActCode A, int MB, int NB, int RUNS>
__device__ __forceinline__ void store_rows(const Params &p, int m, int n, const float (&bias)[RUNS][RUN<TO>], const f32x4 (&acc)[MB][NB]) {
    constexpr int G = MB < 4 ? MB : 4, R = RUN<TO>;
#pragma unroll
    for (int g = 0; g < MB; g += G) {
        TO r[G][RUNS][R];
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int u = 0; u < RUNS; ++u) load_residual(p, m + 16 * (g + i), n + u * 4 * R, r[i][u]);
#pragma unroll
        for (int i = 0; i < G; ++i) {
            if (m + 16 * (g + i) >= p.M) continue;
#pragma unroll
            for (int u = 0; u < RUNS; ++u) {
                if (n + u * 4 * R >= p.N) continue;
                float v[R];
#pragma unroll
                for (int j = 0; j < R; ++j) v[j] = acc[g + i][(u * R + j) >> 2][j & 3];
                finish<R, TO, A>(p, m + 16 * (g + i), n + u * 4 * R, bias[u], r[i][u], v);
            }
        }
    }
}

// Elements [k, k + 8) of a row; zero from K on.
template <typename T>
__device__ __forceinline__ uint4 load_cut(const T *row, int k, int K) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (k >= K) return v;
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

// Rows that may start at any element: a load that is not aligned to 4 bytes takes several times as long (787 x 333 x 1001
// 18.5 us, x 1002 8.0).  Instead 16 bytes are loaded from the 4-byte boundary at or before `at`, the dword behind them is
// taken from the lane that loaded the next 16 bytes of the row or loaded (`tail`), and the five are shifted.  2 of the bytes
// loaded may lie outside of the eight elements, in the same aligned 4 bytes as one of them.
__device__ __forceinline__ uint4 load_floor(const void *at) {
    uint4 v;
    __builtin_memcpy(&v, reinterpret_cast<const void *>(reinterpret_cast<unsigned long long>(at) & ~3ull), 16);
    return v;
}
__device__ __forceinline__ unsigned load_tail(const void *at) {   // the dword behind load_floor's, if it is needed
    const unsigned long long a = reinterpret_cast<unsigned long long>(at);
    return reinterpret_cast<const unsigned *>(a & ~3ull)[a & 2 ? 4 : 3];
}
__device__ __forceinline__ uint4 shift_in(const uint4 &v, unsigned behind, const void *at) {
    const unsigned shift = (static_cast<unsigned>(reinterpret_cast<unsigned long long>(at)) & 2u) * 8u;
    return make_uint4(__builtin_amdgcn_alignbit(v.y, v.x, shift), __builtin_amdgcn_alignbit(v.z, v.y, shift),
                      __builtin_amdgcn_alignbit(v.w, v.z, shift), __builtin_amdgcn_alignbit(behind, v.w, shift));
}
// Elements s on (0 to 8) of eight, and zeros behind them.
__device__ __forceinline__ uint4 drop(uint4 v, int s) {
    if (s & 1) v = make_uint4(__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16),
                              __builtin_amdgcn_alignbit(v.w, v.z, 16), v.w >> 16);
    if (s & 2) v = make_uint4(v.y, v.z, v.w, 0u);
    if (s & 4) v = make_uint4(v.z, v.w, 0u, 0u);
    return s & 8 ? make_uint4(0u, 0u, 0u, 0u) : v;
}

// ---- rows that start anywhere

// A tile of 64 rows by 64 columns a workgroup, four wavefronts of 32 x 32, one slice of 64 elements of the depth at a time
// through LDS, the next one on its way into registers meanwhile.
template <typename T, typename TO, ActCode A, bool ODD>
__global__ __launch_bounds__(256) void staged_kernel(Params p) {
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
    unsigned xt[2] = {}, wt[2] = {};   // ODD: the dword behind, where the next lane does not have it
    auto request = [&](const T *r, int k, int K, uint4 &v, unsigned &tail) {
        if constexpr (!ODD) {
            v = load_cut(r, k, K);
        } else if (k + 8 <= K) {
            v = load_floor(r + k);
            if (q == 7 || k + 16 > K) tail = load_tail(r + k);
        } else {
            v = load_cut(r, k, K);
        }
    };
    // What the loads brought as it goes into LDS.
    auto arrived = [&](const T *r, int k, int K, const uint4 &v, unsigned tail) {
        if constexpr (!ODD) {
            return v;
        } else {
            unsigned behind = __builtin_amdgcn_update_dpp(0, static_cast<int>(v.x), 0x101, 0xf, 0xf, true);   // of the next lane
            if (q == 7 || k + 16 > K) behind = tail;
            return k + 8 <= K ? shift_in(v, behind, r + k) : v;
        }
    };
    auto fetch = [&](int k) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            request(xr[i], k + 8 * q, xok[i] ? p.K : 0, xs[i], xt[i]);
            request(wr[i], k + 8 * q, wok[i] ? p.K : 0, ws[i], wt[i]);
        }
    };
    f32x4 acc[2][2] = {};
    fetch(0);
    for (int k = 0; k < p.K; k += 64) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = (row + 32 * i) * 8 + (q ^ ((row >> 1) & 7));
            tile[0][at] = arrived(xr[i], k + 8 * q, xok[i] ? p.K : 0, xs[i], xt[i]);
            tile[1][at] = arrived(wr[i], k + 8 * q, wok[i] ? p.K : 0, ws[i], wt[i]);
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
    for (int j = 0; j < 2; ++j) {
        const int n = n0 + wn + 16 * j + 4 * (lane >> 4);
        const int m = m0 + wm + (lane & 15);
        float bias[4];
        TO r[2][4];
        load_bias(p, n, bias);
#pragma unroll
        for (int i = 0; i < 2; ++i) load_residual(p, m + 16 * i, n, r[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (m + 16 * i < p.M && n < p.N) finish<4, TO, A>(p, m + 16 * i, n, bias, r[i], v);
        }
    }
}

// ---- tiles staged by transfers to LDS

constexpr unsigned OOB = 0x80000000u;   // byte offset past every row block: the transfer brings zeros

// The tile a workgroup computes.  Every die gets a contiguous run of workgroups; runs go through panels of 8 tile rows column
// by column, so that the 32 CUs of a die share few rows of x and w in their L2 at any time.
struct Tile {
    int m, n, split;
};
__device__ __forceinline__ Tile tile_of(const Params &p, int id) {
    constexpr int PANEL = 8;
    const int tiles = p.tiles_m * p.tiles_n;
    Tile t;
    t.split = fdiv(id, p.d_tiles);
    id -= t.split * tiles;
    const int panel = fdiv(id >> 3, p.d_tiles_n), first = panel * PANEL, rows = min(PANEL, p.tiles_m - first);
    id -= first * p.tiles_n;
    t.n = id / rows;
    t.m = first + id - t.n * rows;
    return t;
}

__device__ __forceinline__ i32x4 make_rsrc(const void *ptr, unsigned bytes) {
    const unsigned long long a = reinterpret_cast<unsigned long long>(ptr);
    return i32x4{__builtin_amdgcn_readfirstlane(static_cast<int>(a)), __builtin_amdgcn_readfirstlane(static_cast<int>((a >> 32) & 0xFFFF)),
                 __builtin_amdgcn_readfirstlane(static_cast<int>(bytes)), 0x00020000};
}
__device__ __forceinline__ unsigned lds_addr(const void *p) {
    return static_cast<unsigned>(reinterpret_cast<unsigned long long>((const __attribute__((address_space(3))) char *)p));
}
// Lane i's 16 bytes at byte offset voff + soff of the buffer go to LDS address base + 16 i.  Issued as assembly so that only
// this kernel's own waits wait for it.  M0 is written undeclared: the compiler keeps nothing in it.
__device__ __forceinline__ void dma16(const i32x4 rsrc, unsigned base, unsigned voff, int soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(base), "v"(voff), "s"(rsrc), "s"(soff)
                 : "memory");
}

// A tile of BM rows by BN columns of y, the depth in slices of 64 through two LDS buffers: while one is multiplied the next
// slice is on its way into the other, and other workgroups of the CU have theirs.  WM x WN wavefronts, each with
// (BM / WM) x (BN / WN) of the tile in 16 x 16 blocks.
//
// Rows of a slice are 128 bytes; chunk c of row r lies at c ^ ((r >> 1) & 7), so that the 16 rows of a fragment read come
// from all 64 banks.  The lane that fills a place fetches the chunk that belongs there.
//
// w is the left operand: a lane's accumulators are four consecutive rows of the block, which are columns of y.  The rows of w
// are stored in the order that makes a lane's columns runs of 16 bytes (column_of): no pass through LDS before the stores.
//
// Measured and left: rings of four buffers (fewer workgroups a CU, 6272 x 1024 x 4096 71 us instead of 56), fragments read
// one half slice ahead (68), slices of 32 (half the rate of transfers), lines brought into L2 five slices ahead (no change).
template <typename T, typename TO, ActCode A, int BM, int BN, int WM, int WN, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN) void tile_kernel(Params p) {
    constexpr int WAVES = WM * WN, MB = BM / WM / 16, NB = BN / WN / 16;
    constexpr int ROWS = BM + BN, PIECES = ROWS / 8 / WAVES;   // transfers of 8 rows a wavefront issues per slice
    constexpr int XP = BM / 8 / WAVES, RUNS = 4 * NB / RUN<TO>;
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "whole pieces");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2][ROWS * 128];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const Tile t = tile_of(p, id);
    const int m0 = t.m * BM, n0 = t.n * BN;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    const int mrows = min(BM, p.M - m0), nrows = min(BN, p.N - n0);
    const i32x4 xs = make_rsrc(static_cast<const T *>(p.x) + static_cast<long long>(m0) * p.ldx, 2u * ((mrows - 1) * p.ldx + p.K));
    const i32x4 ws = make_rsrc(static_cast<const T *>(p.w) + static_cast<long long>(n0) * p.ldw, 2u * ((nrows - 1) * p.ldw + p.K));
    const int k0 = SPLIT ? t.split * p.slices * 64 : 0, k1 = SPLIT ? min(p.K, k0 + p.slices * 64) : p.K;
    const int n_slices = (k1 - k0 + 63) >> 6;

    // piece j of this wavefront: LDS rows 8 (wave + WAVES j) on; x rows first, then w rows
    unsigned voff[PIECES];
    static_assert(WAVES % 2 == 0, "pieces of a wavefront are whole 16 rows apart");
    const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int row = 8 * (wave + WAVES * (j < XP ? j : j - XP)) + (lane >> 3);
        if (j < XP) {
            voff[j] = row < mrows ? static_cast<unsigned>(row * p.ldx + chunk * 8) * 2u : OOB;
        } else {
            const int in = row % (16 * NB), col = row - in + column_of<TO>(in);
            voff[j] = col < nrows ? static_cast<unsigned>(col * p.ldw + chunk * 8) * 2u : OOB;
        }
    }
    const unsigned base = lds_addr(lds);
    auto fetch = [&](int s) {
        const int k = k0 + s * 64;
        const unsigned to = base + (s & 1) * ROWS * 128 + wave * 1024;
        const bool cut = k + 64 > p.K;   // the last slice may be short: its missing chunks are zeros
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            unsigned v = voff[j];
            if (cut && k + 8 * chunk >= p.K) v = OOB;
            dma16(j < XP ? xs : ws, to + (j < XP ? j * WAVES : BM / 8 + (j - XP) * WAVES) * 1024, v, k * 2);
        }
    };
    f32x4 acc[MB][NB] = {};
    // before the first transfer: the waits below count what is on its way
    const int n = n0 + wn * (BN / WN) + (lane >> 4) * RUN<TO>;
    float bias[RUNS][RUN<TO>];
    if (!SPLIT) load_biases<TO>(p, n, bias);
    fetch(0);
    // fragment rows of this lane: the same swizzle for all blocks, since blocks are 16 rows apart
    const int fr = lane & 15, key = (fr >> 1) & 7;
    const int xr = (wm * (BM / WM) + fr) * 128, wr = (BM + wn * (BN / WN) + fr) * 128;
    const int c0 = ((lane >> 4) ^ key) * 16, c1 = ((4 + (lane >> 4)) ^ key) * 16;
    for (int s = 0; s < n_slices; ++s) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < n_slices) fetch(s + 1);
        const unsigned char *buf = lds[s & 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = h ? c1 : c0;
            uint4 a[NB], b[MB];
#pragma unroll
            for (int j = 0; j < NB; ++j) a[j] = *reinterpret_cast<const uint4 *>(buf + wr + j * 2048 + c);
#pragma unroll
            for (int i = 0; i < MB; ++i) b[i] = *reinterpret_cast<const uint4 *>(buf + xr + i * 2048 + c);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mma(a[j], b[i], acc[i][j], T());
        }
    }
    const int m = m0 + wm * (BM / WM) + fr;
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            if (m + 16 * i >= p.M) continue;
            float *y = p.part + (static_cast<size_t>(t.split) * p.M + m + 16 * i) * p.N;
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int at = n + 16 * j;
                if (at + 4 <= p.N && p.N % 4 == 0) {
                    *reinterpret_cast<f32x4 *>(y + at) = acc[i][j];
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (at + c < p.N) y[at + c] = acc[i][j][c];
                }
            }
        }
    } else {
        store_rows<TO, A>(p, m, n, bias, acc);
    }
}

// A tile of BM x BM (256 x 256: 160 KB of LDS, one workgroup a CU) with layouts as above.  Slots hold one operand's slice; x
// of slice s is number 2 s, w number 2 s + 1, number i lies in slot i % 5.  Fragments are read half a slice ahead.  A slice is
// free once the fragments of its second half are in registers; w of slice s + 2 then takes the place of x of slice s, and
// x of slice s + 3 that of w.
template <typename T, typename TO, ActCode A, int BM, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void big_tile_kernel(Params p) {
    constexpr int BN = BM, NBUF = 5;
    constexpr int WAVES = WM * WN, MB = BM / WM / 16, NB = BN / WN / 16;
    constexpr int ROWS = BM + BN, PIECES = ROWS / 8 / WAVES;   // transfers of 8 rows a wavefront issues per slice
    constexpr int XP = BM / 8 / WAVES, RUNS = 4 * NB / RUN<TO>;
    static_assert(BM == BN && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "whole pieces");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NBUF * BM * 128];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const Tile t = tile_of(p, id);
    const int m0 = t.m * BM, n0 = t.n * BN;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    const int mrows = min(BM, p.M - m0), nrows = min(BN, p.N - n0);
    const i32x4 xs = make_rsrc(static_cast<const T *>(p.x) + static_cast<long long>(m0) * p.ldx, 2u * ((mrows - 1) * p.ldx + p.K));
    const i32x4 ws = make_rsrc(static_cast<const T *>(p.w) + static_cast<long long>(n0) * p.ldw, 2u * ((nrows - 1) * p.ldw + p.K));
    const int n_slices = (p.K + 63) >> 6;

    // piece j of this wavefront: LDS rows 8 (wave + WAVES j) on; x rows first, then w rows
    unsigned voff[PIECES];
    static_assert(WAVES % 2 == 0, "pieces of a wavefront are whole 16 rows apart");
    const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int row = 8 * (wave + WAVES * (j < XP ? j : j - XP)) + (lane >> 3);
        if (j < XP) {
            voff[j] = row < mrows ? static_cast<unsigned>(row * p.ldx + chunk * 8) * 2u : OOB;
        } else {
            const int in = row % (16 * NB), col = row - in + column_of<TO>(in);
            voff[j] = col < nrows ? static_cast<unsigned>(col * p.ldw + chunk * 8) * 2u : OOB;
        }
    }
    const unsigned base = lds_addr(lds);
    auto piece = [&](bool w, int j, int s, int slot) {
        const int k = s * 64;
        unsigned v = voff[j + (w ? XP : 0)];
        if (k + 64 > p.K && k + 8 * chunk >= p.K) v = OOB;   // the last slice may be short: its missing chunks are zeros
        dma16(w ? ws : xs, base + slot * BM * 128 + wave * 1024 + j * WAVES * 1024, v, k * 2);
    };
    auto fetch = [&](bool w, int s, int slot) {
#pragma unroll
        for (int j = 0; j < XP; ++j) piece(w, j, s, slot);
    };
    f32x4 acc[MB][NB] = {};
    // fragment rows of this lane: the same swizzle for all blocks, since blocks are 16 rows apart
    const int fr = lane & 15, key = (fr >> 1) & 7;
    const int xr = (wm * (BM / WM) + fr) * 128, wr = (wn * (BN / WN) + fr) * 128;
    const int c0 = ((lane >> 4) ^ key) * 16, c1 = ((4 + (lane >> 4)) ^ key) * 16;
    auto frag = [&](int off) { return *reinterpret_cast<const uint4 *>(lds + off); };
    auto read = [&](uint4 (&a)[NB], uint4 (&b)[MB], int xslot, int wslot, int c) {
#pragma unroll
        for (int j = 0; j < NB; ++j) a[j] = frag(wslot * BM * 128 + wr + c + j * 2048);
#pragma unroll
        for (int i = 0; i < MB; ++i) b[i] = frag(xslot * BM * 128 + xr + c + i * 2048);
    };
    // The products of half a slice; between them the transfers of one operand of a later slice are requested, one at a time:
    // requested at once they fill the queue to memory and hold up the matrix instructions behind them (8192^3 886 us, one
    // at a time 824).
    auto multiply = [&](const uint4 (&a)[NB], const uint4 (&b)[MB], bool fill, bool w, int s, int slot) {
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            if (fill) {
#pragma unroll
                for (int j = i * XP / MB; j < (i + 1) * XP / MB; ++j) piece(w, j, s, slot);
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = mma(a[j], b[i], acc[i][j], T());
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i / 2 < n_slices) fetch(i & 1, i / 2, i);
    uint4 a0[NB], b0[MB], a1[NB], b1[MB];
    if (n_slices >= 2) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(XP * 2) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    read(a0, b0, 0, 1, c0);
    int at = 0;   // slot of x of slice s; w's is the next one
    auto wrap = [](int i) { return i >= NBUF ? i - NBUF : i; };
    for (int s = 0; s < n_slices; ++s) {
        const int wat = wrap(at + 1);
        read(a1, b1, at, wat, c1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(a0, b0, s + 2 < n_slices, false, s + 2, wrap(at + NBUF - 1));
        const int next = wrap(at + 2);
        if (s + 1 < n_slices) {
            // every wavefront has read all of slice s, and slice s + 1 is there; x of slice s + 2 may be on its way
            if (s + 2 < n_slices) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(XP) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            read(a0, b0, next, wrap(next + 1), c0);
        }
        __builtin_amdgcn_sched_barrier(0);
        multiply(a1, b1, s + 2 < n_slices, true, s + 2, at);
        at = next;
    }
    const int n = n0 + wn * (BN / WN) + (lane >> 4) * RUN<TO>;
    float bias[RUNS][RUN<TO>];
    load_biases<TO>(p, n, bias);
    store_rows<TO, A>(p, m0 + wm * (BM / WM) + fr, n, bias, acc);
}

// ---- few rows or few tiles of rows that start anywhere: no LDS in the main loop

// Eight elements each at row, row + 32, ...: lane l has chunk l / 16 of the 32 elements.
template <bool ODD, typename T, int U>
__device__ __forceinline__ void load_run(const T *row, uint4 (&v)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (ODD) v[u] = load_floor(row + 32 * u);
        else __builtin_memcpy(&v[u], row + 32 * u, 16);
    }
}
// The chunk behind a lane's is 16 lanes on, or in the first lanes' next element.
template <typename T, int U>
__device__ __forceinline__ void shift_run(const T *row, uint4 (&v)[U], unsigned tail) {
    const int lane = threadIdx.x & 63, from = ((lane + 16) & 63) * 4;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned give = lane >= 16 ? v[u].x : u + 1 < U ? v[u + 1].x : 0u;
        unsigned behind = __builtin_amdgcn_ds_bpermute(from, static_cast<int>(give));
        if (u + 1 == U && lane >= 48) behind = tail;
        v[u] = shift_in(v[u], behind, row);
    }
}

// 16 MB rows by 16 NB columns of y a workgroup, its wavefronts each with a range of the depth and operands straight from
// memory into the matrix instructions; their sums meet in LDS.  Rows may start at any element.  A wavefront has U steps of 32
// of the depth in flight: what bounds the form is how long memory takes to answer, so everything is asked for at once.  K is
// 8 or more.
template <typename T, typename TO, ActCode A, int MB, int NB, int WAVES, bool ODD>
__global__ __launch_bounds__(64 * WAVES) void direct_kernel(Params p) {
    constexpr int U = 4, ITEMS = MB * NB * 64;
    __shared__ f32x4 sums[WAVES][ITEMS];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int tn = fdiv(id, p.d_tiles_m), tm = id - tn * p.tiles_m;   // the row blocks of a column block next to one another
    const int m0 = tm * 16 * MB, n0 = tn * 16 * NB;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int k0 = wave * p.slices * 32, k1 = min(p.K, k0 + p.slices * 32);
    // item of the sums: four columns of a row
    constexpr int PER = (ITEMS + 64 * WAVES - 1) / (64 * WAVES);
    auto m_of = [&](int item) { return m0 + 16 * ((item >> 6) / NB) + (item & 15); };
    auto n_of = [&](int item) { return n0 + 16 * ((item >> 6) % NB) + 4 * ((item & 63) >> 4); };
    float bias[PER][4];
    TO res[PER][4];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int item = threadIdx.x + u * 64 * WAVES;
        if (item >= ITEMS) continue;
        load_bias(p, n_of(item), bias[u]);
        load_residual(p, m_of(item), n_of(item), res[u]);
    }
    const T *wr[NB], *xr[MB];   // rows behind the last are read as the last; what comes of them is not stored
#pragma unroll
    for (int j = 0; j < NB; ++j)
        wr[j] = static_cast<const T *>(p.w) + static_cast<long long>(min(n0 + 16 * j + (lane & 15), p.N - 1)) * p.ldw;
#pragma unroll
    for (int i = 0; i < MB; ++i)
        xr[i] = static_cast<const T *>(p.x) + static_cast<long long>(min(m0 + 16 * i + (lane & 15), p.M - 1)) * p.ldx;
    f32x4 acc[MB][NB] = {};
    int k = k0 + 8 * (lane >> 4);
    for (; k - 8 * (lane >> 4) + 32 * U <= k1; k += 32 * U) {
        uint4 a[NB][U], b[MB][U];
#pragma unroll
        for (int j = 0; j < NB; ++j) load_run<ODD>(wr[j] + k, a[j]);
#pragma unroll
        for (int i = 0; i < MB; ++i) load_run<ODD>(xr[i] + k, b[i]);
        if constexpr (ODD) {
            unsigned wtail[NB] = {}, xtail[MB] = {};
            if (lane >= 48) {   // the last chunk of the run
#pragma unroll
                for (int j = 0; j < NB; ++j) wtail[j] = load_tail(wr[j] + k + 32 * (U - 1));
#pragma unroll
                for (int i = 0; i < MB; ++i) xtail[i] = load_tail(xr[i] + k + 32 * (U - 1));
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) shift_run(wr[j] + k, a[j], wtail[j]);
#pragma unroll
            for (int i = 0; i < MB; ++i) shift_run(xr[i] + k, b[i], xtail[i]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mma(a[j][u], b[i][u], acc[i][j], T());
    }
    // The rest.  Of a chunk that the row's end cuts the row's last eight elements are loaded instead and moved down; chunks
    // behind the range load whatever is there for nothing.
    const int kb = k - 8 * (lane >> 4);
    if (kb < k1) {
        uint4 a[U][NB], b[U][MB];
        unsigned at[U][NB], bt[U][MB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kb + 32 * u >= k1) continue;
            const int from = min(k + 32 * u, p.K - 8);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if constexpr (ODD) a[u][j] = load_floor(wr[j] + from), at[u][j] = load_tail(wr[j] + from);
                else __builtin_memcpy(&a[u][j], wr[j] + from, 16);
            }
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                if constexpr (ODD) b[u][i] = load_floor(xr[i] + from), bt[u][i] = load_tail(xr[i] + from);
                else __builtin_memcpy(&b[u][i], xr[i] + from, 16);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kb + 32 * u >= k1) continue;
            const int from = min(k + 32 * u, p.K - 8), less = min(max(k + 32 * u + 8 - k1, 0), 8);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if constexpr (ODD) a[u][j] = shift_in(a[u][j], at[u][j], wr[j] + from);
                a[u][j] = drop(a[u][j], less);
            }
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                if constexpr (ODD) b[u][i] = shift_in(b[u][i], bt[u][i], xr[i] + from);
                b[u][i] = drop(b[u][i], less);
            }
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mma(a[u][j], b[u][i], acc[i][j], T());
        }
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[wave][(i * NB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int item = threadIdx.x + u * 64 * WAVES, m = m_of(item), n = n_of(item);
        if (item >= ITEMS || m >= p.M || n >= p.N) continue;
        f32x4 s = sums[0][item];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) s += sums[i][item];
        float v[4] = {s[0], s[1], s[2], s[3]};
        finish<4, TO, A>(p, m, n, bias[u], res[u], v);
    }
}

// ---- few rows or few tiles

// 16 MB rows by 16 NB columns of y a workgroup, its wavefronts each with a range of the depth and a ring of RING slices of 64
// in LDS that nobody else touches: no barrier until their sums meet.  Transfers as in the tile kernels: 8 lanes bring 128
// consecutive bytes of a row, where the matrix instructions' own layout would have 16 lanes ask for 16 rows at once (operands
// straight from memory: 24 x 1024 x 4096 9.1 us instead of 4.9, 197 x 1024 x 4096 17.2 instead of 8.7).
template <typename T, typename TO, ActCode A, int MB, int NB, int WAVES, int RING>
__global__ __launch_bounds__(64 * WAVES) void ring_kernel(Params p) {
    constexpr int PIECES = 2 * (MB + NB), ITEMS = MB * NB * 64, SLOT = PIECES * 1024, LDS = RING * SLOT * WAVES;
    constexpr int SUMS = WAVES * ITEMS * 16;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS > SUMS ? LDS : SUMS];
    const int id = die_block(p.per_die, blockIdx.x);
    if (id >= p.total) return;
    const int tn = fdiv(id, p.d_tiles_m), tm = id - tn * p.tiles_m;   // the row blocks of a column block next to one another
    const int m0 = tm * 16 * MB, n0 = tn * 16 * NB;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int mrows = min(16 * MB, p.M - m0), nrows = min(16 * NB, p.N - n0);
    const i32x4 xs = make_rsrc(static_cast<const T *>(p.x) + static_cast<long long>(m0) * p.ldx, 2u * ((mrows - 1) * p.ldx + p.K));
    const i32x4 ws = make_rsrc(static_cast<const T *>(p.w) + static_cast<long long>(n0) * p.ldw, 2u * ((nrows - 1) * p.ldw + p.K));
    // item of the sums: four columns of a row.  What is added to them is asked for before the first transfer, since the waits
    // below count what is on its way.
    constexpr int PER = (ITEMS + 64 * WAVES - 1) / (64 * WAVES);
    auto m_of = [&](int item) { return m0 + 16 * ((item >> 6) / NB) + (item & 15); };
    auto n_of = [&](int item) { return n0 + 16 * ((item >> 6) % NB) + 4 * ((item & 63) >> 4); };
    float bias[PER][4];
    TO res[PER][4];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int item = threadIdx.x + u * 64 * WAVES;
        if (item >= ITEMS) continue;
        load_bias(p, n_of(item), bias[u]);
        load_residual(p, m_of(item), n_of(item), res[u]);
    }
    const int k0 = wave * p.slices * 64, k1 = min(p.K, k0 + p.slices * 64), n_slices = k1 > k0 ? (k1 - k0 + 63) >> 6 : 0;
    unsigned voff[PIECES];
    const int q = lane & 7;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const int row = 8 * (j < 2 * MB ? j : j - 2 * MB) + (lane >> 3), chunk = q ^ ((row >> 1) & 7);
        voff[j] = row < (j < 2 * MB ? mrows : nrows) ? static_cast<unsigned>(row * (j < 2 * MB ? p.ldx : p.ldw) + chunk * 8) * 2u : OOB;
    }
    unsigned char *mine = lds + wave * RING * SLOT;
    const unsigned base = lds_addr(lds) + wave * RING * SLOT;
    auto fetch = [&](int s, int at) {
        const int k = k0 + s * 64;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            unsigned v = voff[j];
            if (k + 64 > p.K) {
                const int row = 8 * (j < 2 * MB ? j : j - 2 * MB) + (lane >> 3);
                if (k + 8 * (q ^ ((row >> 1) & 7)) >= p.K) v = OOB;
            }
            dma16(j < 2 * MB ? xs : ws, base + at * SLOT + j * 1024, v, k * 2);
        }
    };
#pragma unroll
    for (int i = 0; i < RING; ++i)
        if (i < n_slices) fetch(i, i);
    f32x4 acc[MB][NB] = {};
    const int fr = lane & 15, key = (fr >> 1) & 7;
    const int c0 = ((lane >> 4) ^ key) * 16, c1 = ((4 + (lane >> 4)) ^ key) * 16;
    int at = 0;
    for (int s = 0; s < n_slices; ++s) {
        if (s + RING <= n_slices) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PIECES * (RING - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const unsigned char *buf = mine + at * SLOT + fr * 128;
        uint4 a[2][NB], b[2][MB];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < NB; ++j) a[h][j] = *reinterpret_cast<const uint4 *>(buf + (MB + j) * 2048 + (h ? c1 : c0));
#pragma unroll
            for (int i = 0; i < MB; ++i) b[h][i] = *reinterpret_cast<const uint4 *>(buf + i * 2048 + (h ? c1 : c0));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot is read before it is filled again
        if (s + RING < n_slices) fetch(s + RING, at);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = mma(a[h][j], b[h][i], acc[i][j], T());
        at = at + 1 == RING ? 0 : at + 1;
    }
    __syncthreads();   // nothing is on its way any more
    f32x4 *sums = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[wave * ITEMS + (i * NB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int item = threadIdx.x + u * 64 * WAVES, m = m_of(item), n = n_of(item);
        if (item >= ITEMS || m >= p.M || n >= p.N) continue;
        f32x4 s = sums[item];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) s += sums[i * ITEMS + item];
        float v[4] = {s[0], s[1], s[2], s[3]};
        finish<4, TO, A>(p, m, n, bias[u], res[u], v);
    }
}

// ---- rows laid out anew

// Rows of K elements that start anywhere -> rows of Kp, a multiple of 8, with zeros behind the last element; up to two
// operands.
struct Pack {
    const void *src[2];
    void *dst[2];
    int ld[2];
    int K, Kp, pitch;      // pitch: from row to row of what is written
    int first, items;      // chunks of 8 elements of the first operand and of both
    FastDiv d_chunks;      // by Kp / 8
};
// A thread brings 8 elements; the dword behind unaligned ones comes from its neighbour, as above.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(Pack p) {
    const int i = blockIdx.x * 256 + threadIdx.x, which = i >= p.first, j = i - (which ? p.first : 0);
    const int row = fdiv(j, p.d_chunks), k = (j - row * (p.Kp / 8)) * 8, lane = threadIdx.x & 63;
    const bool in = i < p.items;
    const T *r = static_cast<const T *>(p.src[which]) + (in ? static_cast<long long>(row) * p.ld[which] : 0);
    const bool whole = in && k + 8 <= p.K, last = lane == 63 || k + 16 > p.K;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    unsigned tail = 0;
    if (whole) {
        v = load_floor(r + k);
        if (last) tail = load_tail(r + k);
    }
    unsigned behind = __shfl_down(v.x, 1);
    if (last) behind = tail;
    if (whole) v = shift_in(v, behind, r + k);
    else if (in) v = load_cut(r, k, p.K);
    if (in) *reinterpret_cast<uint4 *>(static_cast<T *>(p.dst[which]) + static_cast<long long>(row) * p.pitch + k) = v;
}

// ---- a depth that several workgroups share

// Adds the partial sums of a tile kernel in the order of their splits.  A thread takes four columns of a row.
template <typename TO, ActCode A>
__global__ __launch_bounds__(256) void join_kernel(Params p) {
    const unsigned i = blockIdx.x * 256u + threadIdx.x, groups = (p.N + 3) / 4;
    const unsigned m = i / groups;
    const int n = static_cast<int>(i - m * groups) * 4;
    if (m >= static_cast<unsigned>(p.M)) return;
    const size_t plane = static_cast<size_t>(p.M) * p.N, at = static_cast<size_t>(m) * p.N + n;
    float v[4] = {}, bias[4];
    TO r[4];
    load_bias(p, n, bias);
    load_residual(p, static_cast<int>(m), n, r);
    if (p.N % 4 == 0) {
        f32x4 s = *reinterpret_cast<const f32x4 *>(p.part + at);
#pragma unroll 8
        for (int k = 1; k < p.splits; ++k) s += *reinterpret_cast<const f32x4 *>(p.part + k * plane + at);
        v[0] = s[0]; v[1] = s[1]; v[2] = s[2]; v[3] = s[3];
    } else {
        for (int k = 0; k < p.splits; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n + j < p.N) v[j] += p.part[k * plane + at + j];
    }
    finish<4, TO, A>(p, static_cast<int>(m), n, bias, r, v);
}

// ---- host side

// Microseconds of the forms, fitted on 256 CUs to 130 shapes of 1 to 8192 rows, 32 to 8192 columns and depths of 64 to 8192
// (what is chosen takes 3 % longer than the fastest form, geometric mean).  A CU takes its share of the workgroups in rounds of
// `resident`; a round costs `round`.  A slice of a tile takes `near` + `far` * (how much of 8 MB the operands are: from the
// caches or from memory) when it has the CU for itself, and `busy` times the workgroups that share the CU if that is longer.
// `finish`: the epilogue of a workgroup.
struct TileCost {
    int bm, bn, resident;
    double round, near, far, busy, finish;
};
constexpr TileCost kTile64 = {64, 64, 5, 0.5, 0.0, 0.46, 0.25, 0.45}, kTile128x64 = {128, 64, 3, 0.0, 0.38, 0.16, 0.325, 1.36},
                   kTile128 = {128, 128, 2, 0.0, 0.44, 0.29, 0.44, 3.2}, kBig = {256, 256, 1, 4.0, 1.35, 0.1, 1.45, 6.0},
                   kStaged = {64, 64, 5, 0.5, 0.50, 0.10, 0.29, 0.46};
// The wavefronts of a ring or direct form work side by side on slices of 64; a round takes as long as its slices one after the
// other or as its operands at `per_kb`, and a workgroup of a direct form no less than `least`.
struct RingCost {
    int mb, nb, waves, resident;
    double round, near, far, per_kb, finish, least;
};
constexpr RingCost kRing11 = {1, 1, 4, 2, 0.1, 0.17, 0.06, 0.0142, 0.36, 0.0}, kRing11W = {1, 1, 16, 1, 0.45, 0.16, 0.60, 0.0072, 0.44, 0.0},
                   kRing12 = {1, 2, 8, 1, 0.32, 0.10, 0.63, 0.0079, 0.61, 0.0}, kRing22 = {2, 2, 4, 2, 0.0, 0.27, 0.09, 0.014, 0.68, 0.0},
                   kRing42 = {4, 2, 4, 1, 0.07, 0.37, 0.09, 0.0175, 1.15, 0.0}, kRing44 = {4, 4, 4, 1, 1.8, 0.06, 0.56, 0.0172, 0.35, 0.0},
                   kDirect = {1, 1, 8, 4, 0.2, 0.31, 0.0, 0.021, 0.0, 0.65}, kDirect22 = {2, 2, 8, 2, 0.0, 0.73, 0.0, 0.027, 0.0, 1.3};
constexpr double kStart = 2.2;
// The launch that joins a shared depth, and its traffic by the megabyte.
constexpr double kJoin = 2.5, kJoinMb = 0.34;
constexpr int kMaxSplit = 8;
// The launch that lays rows out anew, likewise.
constexpr double kPack = 4.5, kPackMb = 0.3;
// What a call of more than one launch takes the host, and each launch of it: a shorter call waits for the host.  (Calls that
// are captured or part of a model do not; the estimate does not know them.)
constexpr double kCall = 3.5, kLaunch = 3.2;

int ceil_div(int a, int b) { return (a + b - 1) / b; }

double from_memory(const MatmulArgs &a) { return std::min(1.0, (1.0 * a.M + a.N) * a.K * 2.0 / 8e6); }

double tile_cost(const TileCost &c, const MatmulArgs &a, int split, int n_cu) {
    const double tiles = 1.0 * ceil_div(a.M, c.bm) * ceil_div(a.N, c.bn) * split;
    const int n = static_cast<int>((tiles + n_cu - 1) / n_cu), slices = ceil_div(ceil_div(a.K, 64), split);
    const double alone = c.near + c.far * from_memory(a);
    auto round = [&](int wgs) { return c.round + slices * std::max(alone, c.busy * wgs); };
    const int rest = n % c.resident;
    double t = kStart + n / c.resident * round(c.resident) + (rest ? round(rest) : 0.0) + c.finish * n;
    if (split > 1) t = std::max(t + kJoin + kJoinMb * 4e-6 * split * a.M * a.N, kCall + 2 * kLaunch);
    return t;
}

double ring_cost(const RingCost &c, const MatmulArgs &a, int n_cu, double slower = 1.0) {
    const double wgs = 1.0 * ceil_div(a.M, 16 * c.mb) * ceil_div(a.N, 16 * c.nb);
    if (wgs > (1 << 20)) return 1e30;   // grids stay below 2^32 threads
    const int n = static_cast<int>((wgs + n_cu - 1) / n_cu), rounds = ceil_div(n, c.resident);
    const double kb = (std::min(a.M, 16 * c.mb) + std::min(a.N, 16 * c.nb)) * (a.K * 2.0 / 1024);
    const double chain = 1.0 * rounds * ceil_div(ceil_div(a.K, 64), c.waves) * (c.near + c.far * from_memory(a));
    return kStart + rounds * c.round + slower * std::max(std::max(chain, n * c.least), n * kb * c.per_kb) + c.finish * n;
}

int padded(int K) { return (K + 7) / 8 * 8; }
// Rows laid out anew start at multiples of 128 bytes, so that a transfer of 128 takes one line: in rows of 4784 elements
// 8042 x 2992 x 4778 took 339 us, in rows of 4800 288.
int pitch(int K) { return (K + 63) / 64 * 64; }
// The transfers to LDS bring aligned 16 bytes.
bool x_aligned(const MatmulArgs &a) { return reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx % 8 == 0 && a.K % 8 == 0; }
bool w_aligned(const MatmulArgs &a) { return reinterpret_cast<uintptr_t>(a.w) % 16 == 0 && a.ldw % 8 == 0 && a.K % 8 == 0; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t pack_x_bytes(const MatmulArgs &a) { return x_aligned(a) ? 0 : round256(2ull * a.M * pitch(a.K)); }
size_t pack_w_bytes(const MatmulArgs &a) { return w_aligned(a) ? 0 : round256(2ull * a.N * pitch(a.K)); }
size_t pack_bytes(const MatmulArgs &a) { return pack_x_bytes(a) + pack_w_bytes(a); }
// Some row of x or w may not start at a multiple of 4 bytes.
bool rows_odd(const MatmulArgs &a) {
    return (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) % 4 != 0 || ((a.ldx | a.ldw) & 1) != 0;
}

template <int BM, int BN>
dim3 set_grid(Params &p) {
    p.tiles_m = ceil_div(p.M, BM);
    p.tiles_n = ceil_div(p.N, BN);
    p.d_tiles = make_fastdiv(p.tiles_m * p.tiles_n);
    p.d_tiles_n = make_fastdiv(p.tiles_n);
    p.d_tiles_m = make_fastdiv(p.tiles_m);
    p.total = p.tiles_m * p.tiles_n * p.splits;
    p.per_die = (p.total + 7) / 8;
    return dim3(8 * p.per_die);
}

template <typename T, typename TO, ActCode A, int MB, int NB, int WAVES>
void launch_direct(Params &p, bool odd, hipStream_t stream) {
    const dim3 grid = set_grid<16 * MB, 16 * NB>(p);
    p.slices = ceil_div(p.K, 32 * WAVES);
    if (odd) direct_kernel<T, TO, A, MB, NB, WAVES, true><<<grid, 64 * WAVES, 0, stream>>>(p);
    else direct_kernel<T, TO, A, MB, NB, WAVES, false><<<grid, 64 * WAVES, 0, stream>>>(p);
}

template <typename T, typename TO, ActCode A, int BM, int BN>
void launch_tile(Params &p, hipStream_t stream) {
    const dim3 grid = set_grid<BM, BN>(p);
    tile_kernel<T, TO, A, BM, BN, 2, 2, false><<<grid, 256, 0, stream>>>(p);
}

template <typename T, typename TO, ActCode A, int MB, int NB, int WAVES, int RING>
void launch_ring(Params &p, hipStream_t stream) {
    const dim3 grid = set_grid<16 * MB, 16 * NB>(p);
    p.slices = ceil_div(ceil_div(p.K, 64), WAVES);
    ring_kernel<T, TO, A, MB, NB, WAVES, RING><<<grid, 64 * WAVES, 0, stream>>>(p);
}

template <typename T, typename TO, ActCode A>
hipError_t launch_split(Params &p, hipStream_t stream) {
    const int slices = ceil_div(p.K, 64);
    p.slices = ceil_div(slices, p.splits);
    p.splits = ceil_div(slices, p.slices);   // none without a slice
    const dim3 grid = set_grid<64, 64>(p);
    tile_kernel<T, float, ActCode::LINEAR, 64, 64, 2, 2, true><<<grid, 256, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const size_t threads = static_cast<size_t>(p.M) * ceil_div(p.N, 4);
    join_kernel<TO, A><<<dim3(static_cast<unsigned>((threads + 255) / 256)), 256, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T, typename TO, ActCode A>
hipError_t launch_act(Params &p, const MatmulChoice &c, bool odd, hipStream_t stream) {
    if (p.splits > 1) return launch_split<T, TO, A>(p, stream);
    switch (c.form) {
        case MatmulForm::RING11: launch_ring<T, TO, A, 1, 1, 4, 4>(p, stream); break;
        case MatmulForm::RING11W: launch_ring<T, TO, A, 1, 1, 16, 2>(p, stream); break;
        case MatmulForm::RING12: launch_ring<T, TO, A, 1, 2, 8, 3>(p, stream); break;
        case MatmulForm::RING22: launch_ring<T, TO, A, 2, 2, 4, 2>(p, stream); break;
        case MatmulForm::RING42: launch_ring<T, TO, A, 4, 2, 4, 3>(p, stream); break;
        case MatmulForm::RING44: launch_ring<T, TO, A, 4, 4, 4, 2>(p, stream); break;
        case MatmulForm::DIRECT: launch_direct<T, TO, A, 1, 1, 8>(p, odd, stream); break;
        case MatmulForm::DIRECT22: launch_direct<T, TO, A, 2, 2, 8>(p, odd, stream); break;
        case MatmulForm::TILE64: launch_tile<T, TO, A, 64, 64>(p, stream); break;
        case MatmulForm::TILE128x64: launch_tile<T, TO, A, 128, 64>(p, stream); break;
        case MatmulForm::TILE128: launch_tile<T, TO, A, 128, 128>(p, stream); break;
        case MatmulForm::BIG: {
            const dim3 grid = set_grid<256, 256>(p);
            big_tile_kernel<T, TO, A, 256, 2, 4><<<grid, 512, 0, stream>>>(p);
            break;
        }
        case MatmulForm::STAGED: {
            set_grid<64, 64>(p);
            if (odd) staged_kernel<T, TO, A, true><<<dim3(p.total), 256, 0, stream>>>(p);
            else staged_kernel<T, TO, A, false><<<dim3(p.total), 256, 0, stream>>>(p);
            break;
        }
    }
    return hipGetLastError();
}

template <typename T, typename TO>
hipError_t launch_types(Params &p, const MatmulChoice &c, bool odd, hipStream_t stream) {
    switch (act_code(p.act)) {
        case ActCode::NORMAL: return launch_act<T, TO, ActCode::NORMAL>(p, c, odd, stream);
        case ActCode::GATE: return launch_act<T, TO, ActCode::GATE>(p, c, odd, stream);
        default: return launch_act<T, TO, ActCode::LINEAR>(p, c, odd, stream);
    }
}

// The form for rows that start at multiples of 16 bytes, and its time.
double choose_aligned(const MatmulArgs &a, int n_cu, size_t ws_bytes, MatmulChoice &best) {
    typedef MatmulForm F;
    double t = 1e30;
    auto consider = [&](F f, int split, double cost) {
        if (cost < t) {
            t = cost;
            best = MatmulChoice{f, split, false};
        }
    };
    // Forms that cannot be the fastest are not looked at: an estimate costs the host 30 ns.
    const double tiles = 1.0 * ceil_div(a.M, 64) * ceil_div(a.N, 64);
    if (a.M <= 64 || tiles <= 3.0 * n_cu) {
        consider(F::RING11, 1, ring_cost(kRing11, a, n_cu));
        consider(F::RING11W, 1, ring_cost(kRing11W, a, n_cu));
        consider(F::RING12, 1, ring_cost(kRing12, a, n_cu));
        if (a.M > 16) {
            consider(F::RING22, 1, ring_cost(kRing22, a, n_cu));
            consider(F::RING42, 1, ring_cost(kRing42, a, n_cu));
            consider(F::RING44, 1, ring_cost(kRing44, a, n_cu));
        }
    }
    if (a.M > 16) consider(F::TILE64, 1, tile_cost(kTile64, a, 1, n_cu));
    if (tiles >= n_cu) {
        consider(F::TILE128x64, 1, tile_cost(kTile128x64, a, 1, n_cu));
        consider(F::TILE128, 1, tile_cost(kTile128, a, 1, n_cu));
    }
    if (tiles >= 4.0 * n_cu) consider(F::BIG, 1, tile_cost(kBig, a, 1, n_cu));
    const size_t plane = 4ull * a.M * a.N;
    if (a.M <= 16 || tiles > 2.0 * n_cu || plane >= (1ull << 32)) return t;
    for (int split = 2; split <= kMaxSplit && split * plane <= ws_bytes && split <= ceil_div(a.K, 64); split *= 2)
        consider(F::TILE64, split, tile_cost(kTile64, a, split, n_cu));
    return t;
}

}  // namespace

MatmulChoice choose_matmul(const MatmulArgs &a, int n_cu) {
    const size_t ws_bytes = a.ws ? a.ws_bytes : 0;
    MatmulChoice best{MatmulForm::STAGED, 1, false};
    if (x_aligned(a) && w_aligned(a)) {
        choose_aligned(a, n_cu, ws_bytes, best);
        return best;
    }
    // odd rows: 787 x 333 x 1001 direct 9.8 us and staged 19.1, x 1002 8.0 and 13.5; 8192 x 2047 x 2047 staged 200 us,
    // 8192 x 2048 x 2046 155
    const bool odd = rows_odd(a);
    double t = (odd ? 1.4 : 1.0) * tile_cost(kStaged, a, 1, n_cu);
    auto consider = [&](const MatmulChoice &c, double cost) {
        if (cost < t) {
            t = cost;
            best = c;
        }
    };
    if (a.K >= 8) consider({MatmulForm::DIRECT, 1, false}, ring_cost(kDirect, a, n_cu, odd ? 1.25 : 1.0));
    if (a.K >= 8) consider({MatmulForm::DIRECT22, 1, false}, ring_cost(kDirect22, a, n_cu, odd ? 1.25 : 1.0));
    const size_t room = pack_bytes(a);
    if (t > kPack && room <= ws_bytes && room < (1ull << 34)) {   // chunks are counted below 2^30
        MatmulArgs b = a;
        b.K = padded(a.K);
        MatmulChoice c{};
        const double cost = kPack + kPackMb * 1e-6 * room + choose_aligned(b, n_cu, ws_bytes - room, c);
        c.pack = true;
        consider(c, std::max(cost, kCall + (c.split > 1 ? 3 : 2) * kLaunch));
    }
    return best;
}

hipError_t launch_matmul(const MatmulArgs &args, const LaunchCtx &ctx, hipStream_t stream, int *launches) {
    MatmulArgs a = args;
    const MatmulChoice c = choose_matmul(a, ctx.n_cu);
    if (launches) *launches = (c.pack ? 1 : 0) + (c.split > 1 ? 2 : 1);
    char *ws = static_cast<char *>(a.ws);
    if (c.pack) {
        Pack k{};
        k.K = a.K;
        k.Kp = padded(a.K);
        k.pitch = pitch(a.K);
        const int chunks = k.Kp / 8;
        k.d_chunks = make_fastdiv(chunks);
        auto add = [&](const void *src, int ld, int rows, size_t bytes) -> const void * {
            if (bytes == 0) return src;
            const int at = k.items == 0 ? 0 : 1;
            k.src[at] = src; k.dst[at] = ws; k.ld[at] = ld;
            k.items += rows * chunks;
            if (at == 0) k.first = k.items;
            ws += bytes;
            return k.dst[at];
        };
        const size_t xb = pack_x_bytes(a), wb = pack_w_bytes(a);
        a.x = add(a.x, a.ldx, a.M, xb);
        a.w = add(a.w, a.ldw, a.N, wb);
        if (xb) a.ldx = k.pitch;
        if (wb) a.ldw = k.pitch;
        a.K = k.Kp;
        const dim3 grid((static_cast<unsigned>(k.items) + 255) / 256);
        if (a.dtype == GPULET_BF16) pack_kernel<__bf16><<<grid, 256, 0, stream>>>(k);
        else pack_kernel<_Float16><<<grid, 256, 0, stream>>>(k);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const bool odd = rows_odd(a);
    Params p{};
    p.x = a.x; p.w = a.w; p.b = a.b; p.r = a.residual; p.y = a.y;
    p.M = a.M; p.N = a.N; p.K = a.K;
    p.ldx = a.ldx; p.ldw = a.ldw; p.ldr = a.ldr; p.ldy = a.ldy;
    p.act = a.act;
    p.splits = c.split;
    p.part = reinterpret_cast<float *>(ws);
    // At the end of a launch the caches of the dies write back what they hold of y.  Small results go past them at once, if they
    // are whole lines: 2048 x 2048 x 512 and the product that reads it back 27.6 us, so 26.3; 500 x 2048 x 512 13.2 and 12.9.
    // Larger ones are left in them: 2156 x 2560 x 640, 11 MB, 38.4 us and past them 44; 9065 x 6272 x 152 113 and 134.
    const int size = a.out_dtype == GPULET_F32 ? 4 : 2;
    p.past = reinterpret_cast<uintptr_t>(a.y) % 128 == 0 && static_cast<long long>(a.ldy) * size % 128 == 0 &&
             1.0 * size * a.M * a.N <= 9e6;
    if (a.dtype == GPULET_BF16)
        return a.out_dtype == GPULET_F32 ? launch_types<__bf16, float>(p, c, odd, stream) : launch_types<__bf16, __bf16>(p, c, odd, stream);
    return a.out_dtype == GPULET_F32 ? launch_types<_Float16, float>(p, c, odd, stream)
                                     : launch_types<_Float16, _Float16>(p, c, odd, stream);
}

size_t matmul_workspace(const MatmulArgs &a) {
    MatmulArgs all = a;
    all.ws = &all;   // any address: nothing is launched
    all.ws_bytes = ~static_cast<size_t>(0);
    size_t bytes = 0;
    for (int n_cu = 8; n_cu <= 256; n_cu += 8) {
        const MatmulChoice c = choose_matmul(all, n_cu);
        bytes = std::max(bytes, (c.pack ? pack_bytes(a) : 0) + (c.split > 1 ? round256(4ull * c.split * a.M * a.N) : 0));
    }
    return bytes;
}

}  // namespace gpulet

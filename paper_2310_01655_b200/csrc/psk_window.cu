// Sliding-window softmax attention (exact attention next to the sketched one: Section 3.2 applies exact weights inside a block; here
// a row sees the `window` rows up to its own, and the first `sinks` rows of its sequence) on the CUDA cores in
// fp32 arithmetic, forward and backward; the cache that goes with it; the checks of all calls.
#include "cc_gemm.cuh"
#include "psk_window.cuh"

#include <math.h>

namespace psk {
namespace win {
namespace {

using namespace cc;

// ---------------------------------------------------------------------------
// Forward and backward by tiles of 64 rows (or keys), 128 threads to a CTA, three CTAs to an SM; the forward in steps of 64 keys, the backward in
// steps of 32.  Bound: fp32 FMA rate, and the latency of what stands between the products: more, smaller threads win (24 heads x 2048
// rows, window 256, one sink, forward / query side / key side: 143 / 201 / 252 us; 64 threads with 8 x 8 values each, at most 255 registers
// and so 6 to 8 warps to an SM, 198 / 247 / 388).
// ---------------------------------------------------------------------------
constexpr int kTile = 64, kThreads = 128;

// ROWS rows x 64 columns from row r0 into [ROWS][kLd] fp32, zeros from row `end` on.  fp32: asynchronous copies, all on their way at once (through
// registers, in batches of four: the forward 13 % slower); cp_wait<> before the barrier in front of their use.
template <int ROWS = kTile, typename T>
__device__ __forceinline__ void load_tile(float* dst, const T* src, int64_t stride, int r0, int end) {
    constexpr int V = 16 / sizeof(T), PerRow = 64 / V;
    if constexpr (sizeof(T) == 4) {
#pragma unroll 8
        for (int e = threadIdx.x; e < ROWS * PerRow; e += kThreads) {
            const int r = e / PerRow, c = e % PerRow * V, bytes = r0 + r < end ? 16 : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst + r * kLd + c)),
                         "l"(src + (bytes ? (int64_t)(r0 + r) * stride + c : 0)), "r"(bytes) : "memory");
        }
        cp_commit();
        return;
    }
#pragma unroll 4
    for (int e = threadIdx.x; e < ROWS * PerRow; e += kThreads) {
        const int r = e / PerRow, c = e % PerRow * V;
        float* d = dst + r * kLd + c;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r0 + r < end) u = *reinterpret_cast<const uint4*>(src + (int64_t)(r0 + r) * stride + c);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(d + 2 * i) = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    } else {
        uint32_t u, v;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(b), "f"(a));
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(d), "f"(c));
        *reinterpret_cast<uint2*>(p) = make_uint2(u, v);
    }
}
// Half of a 64 x 64 accumulator in the outer form: the thread's 8 rows and 4 columns of one half (32 columns) each.
struct HalfAcc {
    f2 s[4][2], x[4][2];              // straight / swapped column pairs
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 2; ++q) s[p][q] = x[p][q] = 0ull;
    }
    // += At^T B over k < K: At [K][kLd] (64 rows), B [K][kLd], from the thread's columns on
    __device__ __forceinline__ void add(const float* At, const float* B, int K, int ry) {
#pragma unroll 4
        for (int k = 0; k < K; ++k) {
            f2 a[4];
            load_rows8(a, At + k * kLd + 8 * ry);
            const F22 b = lds22(B + k * kLd);
            const f2 c[2] = {b.x, b.y};
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f2 sw = swap2(c[q]);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    s[p][q] = fma2(a[p], c[q], s[p][q]);
                    x[p][q] = fma2(a[p], sw, x[p][q]);
                }
            }
        }
    }
    __device__ __forceinline__ float at(int i, int j) const {
        const f2 v = ((i ^ j) & 1) ? x[i / 2][j / 2] : s[i / 2][j / 2];
        return (i & 1) ? hi2(v) : lo2(v);
    }
    // Row i times f; false if one of the half's 32 values is not finite (the same in its 8 lanes).
    __device__ __forceinline__ bool row(int i, float f, float (&o)[4]) const {
        bool fine = true;
#pragma unroll
        for (int j = 0; j < 4; ++j) { o[j] = at(i, j) * f; fine = fine && finite(o[j]); }
        const unsigned all = __ballot_sync(0xffffffffu, fine);
        return (all >> (threadIdx.x % 32 / 8 * 8) & 0xffu) == 0xffu;
    }
};
// d[i][j] = sum_{k < 64} A[ry + 8 i][k] B[cx + 8 j][k], four rows by four columns.
__device__ __forceinline__ void dot_quarter(f2 (&d)[4][4], const float* A, const float* B, int ry, int cx) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) d[i][j] = 0ull;
    const float *a0 = A + ry * kLd, *b0 = B + cx * kLd;
#pragma unroll 4
    for (int k = 0; k < 64; k += 4) {
        F22 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = lds22(a0 + 8 * i * kLd + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const F22 b = lds22(b0 + 8 * j * kLd + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                d[i][j] = fma2(a[i].x, b.x, d[i][j]);
                d[i][j] = fma2(a[i].y, b.y, d[i][j]);
            }
        }
    }
}
template <typename T> __device__ __forceinline__ void store_row(T* p, const float (&o)[4]) { store4(p, o[0], o[1], o[2], o[3]); }
template <typename T>
__device__ __forceinline__ void zero_rows(T* p, int64_t stride, int r0, int end) {
    for (int e = threadIdx.x; e < kTile * 16; e += kThreads)
        if (r0 + e / 16 < end) store4(p + (int64_t)(r0 + e / 16) * stride + e % 16 * 4, 0.f, 0.f, 0.f, 0.f);
}

// Do the `rows` rows from i_first on see all of the keys k0 .. k0 + tile - 1?
__device__ __forceinline__ bool sees_all(int i_first, int rows, int k0, int tile, int window, int sinks) {
    return k0 + tile - 1 <= i_first && (window_start(i_first + rows - 1, window) <= k0 || sinks - k0 >= tile);
}

struct Place { int b, h, row0, len; };
__device__ __forceinline__ Place place_of(const WinArgs& a, int heads) {
    const int tiles = (a.n + kTile - 1) / kTile, bh = blockIdx.x / tiles;
    Place p;
    p.b = bh / heads;
    p.h = bh % heads;
    p.row0 = (int)(blockIdx.x % tiles) * kTile;
    p.len = length_of(a, p.b);
    return p;
}

// (on its own: what it needs is worked out again, not kept in registers over the forward's loop)
template <typename T>
__device__ __noinline__ void redo_out_rows(const WinArgs& a, const int* bad) {
    const Place z = place_of(a, a.H);
    const int64_t at = z.b * a.qb + z.h * a.qh, from = z.b * a.kb + z.h / a.G * a.kh;
    const T *K = (const T*)a.K + from, *V = (const T*)a.V + from;
    for (int r = threadIdx.x / 32; r < kTile && z.row0 + r < z.len; r += kThreads / 32)
        if (bad[r] && row_tainted(K, V, a.kn, z.row0 + r, a.window, a.sinks, z.len)) {
            const int64_t row = at + (z.row0 + r) * a.qn;
            st2((T*)a.out + row + 2 * (threadIdx.x % 32), redo_out_row((const T*)a.Q + row, K, V, a.kn, z.row0 + r, a.window, a.sinks, a.c));
        }
}

constexpr size_t kFwdSmem = 4 * kUnit * sizeof(float);

template <typename T>
__global__ void __launch_bounds__(kThreads, 3)
win_fwd_kernel(const __grid_constant__ WinArgs a) {
    pdl_sync();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    extern __shared__ float sm[];
    __shared__ float s_al[kTile], s_inv[kTile];
    __shared__ int s_nan[kTile], s_bad[kTile];
    float *sQ = sm, *sK = sm + kUnit, *sV = sm + 2 * kUnit, *sP = sm + 3 * kUnit;
    const int tid = threadIdx.x, half = tid / 64, ry = tid % 64 / 8, cx = tid % 8, col = 32 * half + 4 * cx;
    const Place pl = place_of(a, a.H);
    const T* Q = (const T*)a.Q + pl.b * a.qb + pl.h * a.qh;
    const int64_t koff = pl.b * a.kb + pl.h / a.G * a.kh;
    const T *K = (const T*)a.K + koff, *V = (const T*)a.V + koff;
    T* O = (T*)a.out + pl.b * a.qb + pl.h * a.qh;
    float* lse = a.lse + ((int64_t)pl.b * a.H + pl.h) * a.n;
    const int row0 = pl.row0, len = pl.len, n_end = row0 + kTile < a.n ? row0 + kTile : a.n, end = row0 + kTile < len ? row0 + kTile : len;
    // rows behind the sequence's end
    zero_rows(O + (int64_t)(end > row0 ? end - row0 : 0) * a.qn, a.qn, row0, n_end - (end > row0 ? end - row0 : 0));
    for (int r = (end > row0 ? end : row0) + tid; r < n_end; r += kThreads) lse[r] = neg_inf();
    if (end <= row0) return;
    load_tile(sQ, Q, a.qn, row0, end);
    // scores: rows ry + 32 half + 8 i, columns cx + 8 j
    float m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { m[i] = neg_inf(); l[i] = 0.f; }
    HalfAcc acc;
    acc.zero();
    const KeyTiles kt = key_tiles(row0, end - 1, a.window, a.sinks, kTile);
    const int steps = kt.count();
    load_tile(sK, K, a.kn, kt.at(0) * kTile, len);
    load_tile(sV, V, a.kn, kt.at(0) * kTile, len);
    for (int x = 0; x < steps; ++x) {
        const int k0 = kt.at(x) * kTile;
        cp_wait<1>();                                     // the keys; the values may still be on their way
        __syncthreads();
        const bool whole = sees_all(row0, kTile, k0, kTile, a.window, a.sinks);
        {
            f2 d[4][8];
            dot_half<kLd, kLd>(d, sQ, sK, 16, half, ry, cx);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ry + 32 * half + 8 * i;
                float p[8], top = m[i];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float s = sum2(d[i][j]) * a.c;
                    p[j] = whole || sees(row0 + r, k0 + cx + 8 * j, a.window, a.sinks) ? s : neg_inf();
                    top = fmaxf(top, p[j]);
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float base = top == neg_inf() ? 0.f : top, alpha = exp2_approx(m[i] - base);
                m[i] = top;
                l[i] *= alpha;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = exp2_approx(p[j] - base);
                    l[i] += p[j];
                    sP[(cx + 8 * j) * kLd + r] = p[j];
                }
                if (cx == 0) s_al[r] = alpha;
            }
        }
        cp_wait<0>();                                     // the values
        __syncthreads();                                  // everyone has read the keys
        if (x + 1 < steps) load_tile(sK, K, a.kn, kt.at(x + 1) * kTile, len);
#pragma unroll
        for (int p2 = 0; p2 < 4; ++p2) {
            const f2 al = *reinterpret_cast<const f2*>(s_al + 8 * ry + 2 * p2);
#pragma unroll
            for (int q = 0; q < 2; ++q) { acc.s[p2][q] = mul2(acc.s[p2][q], al); acc.x[p2][q] = mul2(acc.x[p2][q], al); }
        }
        acc.add(sP, sV + col, kTile, ry);
        __syncthreads();
        if (x + 1 < steps) load_tile(sV, V, a.kn, kt.at(x + 1) * kTile, len);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
        if (cx == 0) {
            const int r = ry + 32 * half + 8 * i;
            const float v = (m[i] + log2f(l[i])) * kLn2;
            s_inv[r] = 1.f / l[i];
            s_nan[r] = !finite(v);                        // (then neither is the row: NaN)
            s_bad[r] = 0;
            if (row0 + r < end) lse[row0 + r] = v;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = out_row(ry, i);
        float o[4];
        const bool fine = acc.row(i, s_inv[r], o);
        if (row0 + r < end) store_row(O + (int64_t)(row0 + r) * a.qn + col, o);
        if (!fine && !s_nan[r]) s_bad[r] = 1;
    }
    __syncthreads();
    redo_out_rows<T>(a, s_bad);
}

// Keys (query side) or query rows (key side) of a step of the backward.  32: less of a window's edges is computed for nothing, and three CTAs fit
// on the key side (us with 32 / 64: window 256 as above 201 / 218 and 252 / 266; causal, 4 heads x 4096: 779 / 787 and 921 / 893).
constexpr int kStep = 32;
constexpr size_t kDqSmem = 4 * kUnit * sizeof(float);

// The gradient of 64 query rows; their statistics on the way, which the key side reads.
template <typename T>
__global__ void __launch_bounds__(kThreads, 3)
win_dq_kernel(const __grid_constant__ WinArgs a) {
    pdl_sync();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    extern __shared__ float sm[];
    __shared__ float s_D[kTile], s_lse[kTile];
    __shared__ int s_bad[kTile];
    float *sQ = sm, *sG = sm + kUnit, *sK = sm + 2 * kUnit, *sV = sK + 2 * kStep * kLd, *sP = sV + kStep * kLd;
    const int tid = threadIdx.x, half = tid / 64, ry = tid % 64 / 8, cx = tid % 8, col = 32 * half + 4 * cx;
    const Place pl = place_of(a, a.H);
    const int64_t qoff = pl.b * a.qb + pl.h * a.qh, koff = pl.b * a.kb + pl.h / a.G * a.kh, soff = ((int64_t)pl.b * a.H + pl.h) * a.n;
    const T *Q = (const T*)a.Q + qoff, *dO = (const T*)a.dO + qoff, *O = (const T*)a.O + qoff, *K = (const T*)a.K + koff, *V = (const T*)a.V + koff;
    T* dQ = (T*)a.dQ + qoff;
    const int row0 = pl.row0, len = pl.len, n_end = row0 + kTile < a.n ? row0 + kTile : a.n, end = row0 + kTile < len ? row0 + kTile : len;
    zero_rows(dQ + (int64_t)(end > row0 ? end - row0 : 0) * a.qn, a.qn, row0, n_end - (end > row0 ? end - row0 : 0));
    for (int r = (end > row0 ? end : row0) + tid; r < n_end; r += kThreads) a.stat_l[soff + r] = a.stat_d[soff + r] = 0.f;
    if (end <= row0) return;
    load_tile(sQ, Q, a.qn, row0, end);
    load_tile(sG, dO, a.qn, row0, end);
    load_tile(sK, O, a.qn, row0, end);
    cp_wait<0>();
    __syncthreads();
    if (tid < kTile) {
        float D = 0.f;
#pragma unroll 8
        for (int c = 0; c < 64; ++c) D = fmaf(sG[tid * kLd + c], sK[tid * kLd + c], D);
        s_D[tid] = D;
        s_lse[tid] = row0 + tid < end ? a.lse_in[soff + row0 + tid] * kLog2e : 0.f;
        if (row0 + tid < end) { a.stat_l[soff + row0 + tid] = -s_lse[tid]; a.stat_d[soff + row0 + tid] = -D; }
    }
    HalfAcc acc;
    acc.zero();
    const KeyTiles kt = key_tiles(row0, end - 1, a.window, a.sinks, kStep);
    const int steps = kt.count();
    __syncthreads();
    load_tile<kStep>(sK, K, a.kn, kt.at(0) * kStep, len);
    load_tile<kStep>(sV, V, a.kn, kt.at(0) * kStep, len);
    for (int x = 0; x < steps; ++x) {
        const int k0 = kt.at(x) * kStep;
        const float* keys = sK + (x & 1) * kStep * kLd;
        cp_wait<0>();
        __syncthreads();
        if (x + 1 < steps) load_tile<kStep>(sK + (~x & 1) * kStep * kLd, K, a.kn, kt.at(x + 1) * kStep, len);
        const bool whole = sees_all(row0, kTile, k0, kStep, a.window, a.sinks);
        // rows: keys ry + 8 i; columns: queries 32 half + cx + 8 j
        float ds[4][4];
        f2 d[4][4];
        dot_quarter(d, keys, sQ + 32 * half * kLd, ry, cx);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = 32 * half + cx + 8 * j;
            const float base = s_lse[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool v = whole || sees(row0 + r, k0 + ry + 8 * i, a.window, a.sinks);
                ds[i][j] = v ? exp2_approx(fmaf(sum2(d[i][j]), a.c, -base)) : 0.f;
            }
        }
        dot_quarter(d, sV, sG + 32 * half * kLd, ry, cx);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = 32 * half + cx + 8 * j;
            const float D = s_D[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool v = whole || sees(row0 + r, k0 + ry + 8 * i, a.window, a.sinks);
                sP[(ry + 8 * i) * kLd + r] = v ? ds[i][j] * (sum2(d[i][j]) - D) : 0.f;
            }
        }
        __syncthreads();                                  // (and everyone has read the values)
        if (x + 1 < steps) load_tile<kStep>(sV, V, a.kn, kt.at(x + 1) * kStep, len);
        acc.add(sP, keys + col, kStep, ry);
    }
    if (tid < kTile) s_bad[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = out_row(ry, i);
        float o[4];
        const bool nan = s_lse[r] != s_lse[r] || s_D[r] != s_D[r], fine = acc.row(i, a.scale, o) || nan;      // (nan: then so is the row)
        if (row0 + r < end) store_row(dQ + (int64_t)(row0 + r) * a.qn + col, o);
        if (!fine) s_bad[r] = 1;
    }
    __syncthreads();
    for (int r = tid / 32; row0 + r < end && r < kTile; r += kThreads / 32)
        if (s_bad[r] && row_tainted(K, V, a.kn, row0 + r, a.window, a.sinks, len)) {
            const int64_t at = (int64_t)(row0 + r) * a.qn;
            st2(dQ + at + 2 * (tid % 32), redo_dq_row(Q + at, dO + at, K, V, a.kn, row0 + r, a.window, a.sinks, a.c, a.scale, make_float2(s_lse[r], s_D[r])));
        }
}

constexpr size_t kDkvSmem = 4 * kUnit * sizeof(float);

// The gradients of 64 keys and values: sums over the query rows that see them, head by head of those that share them (a fixed order).
// SPLIT 1: there are items that are parts of the sinks' tiles; 2: that, or key heads in several
template <typename T, int SPLIT>
__global__ void __launch_bounds__(kThreads, 3)
win_dkv_kernel(const __grid_constant__ WinArgs a) {
    pdl_sync();
    const int hs = SPLIT == 2 ? a.hs : 1;
    extern __shared__ float sm[];
    __shared__ float s_D[kStep], s_lse[kStep];
    __shared__ int s_bad[kTile];
    float *sK = sm, *sV = sm + kUnit, *sQ = sm + 2 * kUnit, *sG = sQ + kStep * kLd, *sP = sm + 3 * kUnit, *sS = sP + kStep * kLd;
    const int tid = threadIdx.x, half = tid / 64, ry = tid % 64 / 8, cx = tid % 8, col = 32 * half + 4 * cx;
    const int tiles = (a.n + kTile - 1) / kTile;
    const KeyItem it = key_item(a, blockIdx.x, kTile, [&](int x) { return x / tiles; }, [&](int x) { return x / a.Hkv; },
                                [&](int x) { return x / a.parts; });
    const int64_t koff = it.b * a.kb + it.h / hs * a.kh;
    T *dK = (T*)a.dK + koff, *dV = (T*)a.dV + koff;
    const int key0 = it.key0, len = it.len, n_end = key0 + kTile < a.n ? key0 + kTile : a.n, end = key0 + kTile < len ? key0 + kTile : len;
    if ((SPLIT == 0 || it.part <= 0) && hs == 1) {
        const int none = end > key0 ? end - key0 : 0;
        zero_rows(dK + (int64_t)none * a.kn, a.kn, key0, n_end - none);
        zero_rows(dV + (int64_t)none * a.kn, a.kn, key0, n_end - none);
    }
    if (it.empty()) return;
    const int row_end = it.end(a, kTile);
    load_tile(sK, (const T*)a.K + koff, a.kn, key0, end);
    load_tile(sV, (const T*)a.V + koff, a.kn, key0, end);
    HalfAcc ak, av;
    ak.zero();
    av.zero();
    for (int g = 0; g < a.G; ++g) {
        const int h = it.h * a.G + g;
        const int64_t qoff = it.b * a.qb + h * a.qh, soff = ((int64_t)it.b * a.H + h) * a.n;
        const T *Q = (const T*)a.Q + qoff, *dO = (const T*)a.dO + qoff;
        for (int i0 = it.begin; i0 < row_end; i0 += kStep) {
            __syncthreads();
            load_tile<kStep>(sQ, Q, a.qn, i0, len);
            load_tile<kStep>(sG, dO, a.qn, i0, len);
            if (tid < 2 * kStep) {
                const int si = i0 + tid % kStep;
                (tid < kStep ? s_lse : s_D)[tid % kStep] = si < len ? -(tid < kStep ? a.stat_l : a.stat_d)[soff + si] : 0.f;
            }
            cp_wait<0>();
            __syncthreads();
            const bool whole = i0 + kStep <= len && key0 + kTile - 1 <= i0 && (i0 + kStep - 1 - key0 < a.window || key0 + kTile <= a.sinks);
            // rows: queries ry + 8 i; columns: keys 32 half + cx + 8 j
            f2 d[4][4];
            float p[4][4];
            dot_quarter(d, sQ, sK + 32 * half * kLd, ry, cx);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ry + 8 * i;
                const float base = s_lse[r];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = 32 * half + cx + 8 * j;
                    const bool v = whole || (i0 + r < len && sees(i0 + r, key0 + c, a.window, a.sinks));
                    p[i][j] = v ? exp2_approx(fmaf(sum2(d[i][j]), a.c, -base)) : 0.f;
                    sP[r * kLd + c] = p[i][j];
                }
            }
            dot_quarter(d, sG, sV + 32 * half * kLd, ry, cx);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ry + 8 * i;
                const float D = s_D[r];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = 32 * half + cx + 8 * j;
                    const bool v = whole || (i0 + r < len && sees(i0 + r, key0 + c, a.window, a.sinks));
                    sS[r * kLd + c] = v ? p[i][j] * (sum2(d[i][j]) - D) : 0.f;
                }
            }
            __syncthreads();
            av.add(sP, sG + col, kStep, ry);
            ak.add(sS, sQ + col, kStep, ry);
        }
    }
    if (tid < kTile) s_bad[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = out_row(ry, i);
        float k[4], v[4];
        const bool fk = ak.row(i, a.scale, k), fv = av.row(i, 1.f, v), fine = fk && fv;
        // (a part's sums stay as they are: each of its pairs counts)
        if (key0 + r < end) {
            if ((SPLIT == 0 || it.part <= 0) && hs == 1) {
                store_row(dK + (int64_t)(key0 + r) * a.kn + col, k);
                store_row(dV + (int64_t)(key0 + r) * a.kn + col, v);
            } else if ((SPLIT == 0 || it.part <= 0)) {
                store_row(sum_row(a, it.b, it.h, 0, key0 + r) + col, k);
                store_row(sum_row(a, it.b, it.h, 1, key0 + r) + col, v);
            }
            if (SPLIT > 0 && it.part >= 0 && r < a.sinks) {
                store_row(partial_row(a, it.b, it.h, it.part, 0, r) + col, k);
                store_row(partial_row(a, it.b, it.h, it.part, 1, r) + col, v);
            }
        }
        if (!fine && (SPLIT == 0 || it.part <= 0)) s_bad[r] = 1;
    }
    __syncthreads();
    for (int r = tid / 32; key0 + r < end && r < kTile; r += kThreads / 32)
        if (s_bad[r] && key_tainted<T>(a, it.b, it.h, key0 + r, len, it.stop)) {
            const int c = 2 * (tid % 32);
            const bool sum = SPLIT > 0 && it.part == 0 && r < a.sinks;
            const KeyRow k = redo_dkv_row<T>(a, it.b, it.h, key0 + r, len, sum ? row_end : len);
            if (hs == 1) {
                st2(dK + (int64_t)(key0 + r) * a.kn + c, k.dk);
                st2(dV + (int64_t)(key0 + r) * a.kn + c, k.dv);
            } else {
                st2(sum_row(a, it.b, it.h, 0, key0 + r) + c, k.dk);
                st2(sum_row(a, it.b, it.h, 1, key0 + r) + c, k.dv);
            }
            if (sum) {
                st2(partial_row(a, it.b, it.h, 0, 0, r) + c, k.dk);
                st2(partial_row(a, it.b, it.h, 0, 1, r) + c, k.dv);
            }
        }
}

// The sinks' gradients from their parts.
template <typename T>
__global__ void __launch_bounds__(256)
win_sink_sum_kernel(const __grid_constant__ WinArgs a) {
    pdl_sync();
    const int b = blockIdx.x / a.Hkv, hk = blockIdx.x % a.Hkv, len = length_of(a, b), rows = a.sinks < len ? a.sinks : len;
    const int64_t koff = b * a.kb + hk * a.kh;
    const int e = blockIdx.y * 256 + threadIdx.x;
    if (e < rows * 128) {
        const int which = e / (rows * 64), j = e / 64 % rows, c = e % 64;
        float t = partial_row(a, b, hk, 0, which, j)[c];
#pragma unroll 8
        for (int q = 0; q < a.parts && a.split_row + q * a.part_rows < len; ++q) t += partial_row(a, b, hk, q + 1, which, j)[c];
        stf((T*)(which ? a.dV : a.dK) + koff + (int64_t)j * a.kn + c, t);
    }
}

// The gradients of keys and values whose query heads were dealt to several (the sinks' from their parts): four columns of a row to a thread.
template <typename T>
__global__ void __launch_bounds__(256)
win_head_sum_kernel(const __grid_constant__ WinArgs a) {
    pdl_sync();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;             // [B, real key head, dK/dV, row, 16 x 4 columns]
    const int c = (int)(e % 16) * 4;
    const int64_t row = e / 16;
    const int j = (int)(row % a.n), which = (int)(row / a.n % 2), heads = a.Hkv / a.hs;
    const int64_t bh = row / a.n / 2;
    if (bh >= (int64_t)a.B * heads) return;
    const int b = (int)(bh / heads), hk = (int)(bh % heads), len = length_of(a, b);
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float* p) {
        const float4 v = *reinterpret_cast<const float4*>(p + c);
        t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
    };
    if (j < len)
        for (int h = hk * a.hs; h < (hk + 1) * a.hs; ++h) {
            if (a.parts == 0 || j >= a.sinks) { add(sum_row(a, b, h, which, j)); continue; }
            add(partial_row(a, b, h, 0, which, j));
            for (int q = 0; q < a.parts && a.split_row + q * a.part_rows < len; ++q) add(partial_row(a, b, h, q + 1, which, j));
        }
    store4((T*)(which ? a.dV : a.dK) + b * a.kb + hk * a.kh + (int64_t)j * a.kn + c, t.x, t.y, t.z, t.w);
}

template <typename Kern>
cudaError_t launch_rows(const char* name, Kern kern, size_t smem, unsigned grid, const WinArgs& a, cudaStream_t s) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    prof_begin(name, s);
    launch_pdl(kern, dim3(grid), dim3(kThreads), smem, s, a);
    prof_end(s);
    return cudaGetLastError();
}
template <typename T>
cudaError_t cc_window_fwd(const WinArgs& a, cudaStream_t s) {
    const unsigned tiles = (unsigned)((a.n + kTile - 1) / kTile);
    return launch_rows("win_fwd_kernel", win_fwd_kernel<T>, kFwdSmem, tiles * a.B * a.H, a, s);
}
template <typename T>
cudaError_t cc_window_bwd(const WinArgs& a, const WinArgs& k, cudaStream_t s) {
    const unsigned tiles = (unsigned)((a.n + kTile - 1) / kTile);
    const cudaError_t e = launch_rows("win_dq_kernel", win_dq_kernel<T>, kDqSmem, tiles * a.B * a.H, a, s);
    return e != cudaSuccess ? e : launch_rows("win_dkv_kernel", k.hs > 1 ? win_dkv_kernel<T, 2> : k.parts > 0 ? win_dkv_kernel<T, 1> : win_dkv_kernel<T, 0>, kDkvSmem, (tiles + k.parts) * k.B * k.Hkv, k, s);
}
cudaError_t key_sums(const WinArgs& a, bool half, cudaStream_t s) {
    if (a.hs > 1) {
        const int64_t grid = ((int64_t)a.B * (a.Hkv / a.hs) * a.n * 32 + 255) / 256;
        prof_begin("win_head_sum_kernel", s);
        if (half) launch_pdl(win_head_sum_kernel<bf16>, dim3((unsigned)grid), dim3(256), 0, s, a);
        else launch_pdl(win_head_sum_kernel<float>, dim3((unsigned)grid), dim3(256), 0, s, a);
        prof_end(s);
        return cudaGetLastError();
    }
    if (a.parts == 0) return cudaSuccess;
    prof_begin("win_sink_sum_kernel", s);
    if (half) launch_pdl(win_sink_sum_kernel<bf16>, dim3(a.B * a.Hkv, (a.sinks + 1) / 2), dim3(256), 0, s, a);
    else launch_pdl(win_sink_sum_kernel<float>, dim3(a.B * a.Hkv, (a.sinks + 1) / 2), dim3(256), 0, s, a);
    prof_end(s);
    return cudaGetLastError();
}

}  // namespace

// ---- host ----

int check_common(const psk_window_shape* sh) {
    if (sh == nullptr) return PSK_ERR_INVALID_ARG;
    if (sh->dtype != PSK_F32 && sh->dtype != PSK_BF16) return PSK_ERR_INVALID_ARG;
    if (sh->path < PSK_PATH_AUTO || sh->path > PSK_PATH_TENSOR_CORES) return PSK_ERR_INVALID_ARG;
    if (!(sh->scale > 0.f) || isinf(sh->scale * kLog2e)) return PSK_ERR_INVALID_ARG;      // (scores are kept times log2(e))
    if (sh->B <= 0 || sh->H <= 0 || sh->Hkv <= 0 || sh->H % sh->Hkv != 0) return PSK_ERR_SHAPE;
    if (sh->window <= 0 || sh->sinks < 0) return PSK_ERR_SHAPE;
    if ((int64_t)sh->B * sh->H >= (int64_t)1 << 31) return PSK_ERR_SHAPE;
    return sh->h == 64 ? PSK_OK : PSK_ERR_UNSUPPORTED;
}
// [B,H,n,64] with these strides: rows that do not overlap, all on 16 bytes.  (The stride of an extent of 1 is not looked at.)
static int check_strides(int64_t B, int64_t H, int64_t n, int64_t sb, int64_t sh, int64_t sn, int esz) {
    const int64_t e[3] = {B, H, n}, s[3] = {sb, sh, sn};
    bool used[3] = {false, false, false};
    int64_t end = 64;
    for (int k = 0; k < 3; ++k) {
        int at = -1;
        for (int i = 0; i < 3; ++i)
            if (!used[i] && e[i] > 1 && (at < 0 || s[i] < s[at])) at = i;
        if (at < 0) break;
        used[at] = true;
        if (s[at] < end || s[at] >= (int64_t)1 << 39 || s[at] > ((int64_t)1 << 44) / (e[at] - 1)) return PSK_ERR_SHAPE;      // (no memory is that large)
        if (s[at] * esz % 16) return PSK_ERR_ALIGN;
        end += s[at] * (e[at] - 1);
    }
    return PSK_OK;
}
int check_rows(const psk_window_shape* sh) {
    int st = check_common(sh);
    if (st != PSK_OK) return st;
    if (sh->n <= 0 || (int64_t)sh->B * sh->H * sh->n >= (int64_t)1 << 31) return PSK_ERR_SHAPE;
    if (sh->path == PSK_PATH_TENSOR_CORES && sh->dtype != PSK_BF16) return PSK_ERR_UNSUPPORTED;
    const int esz = sh->dtype == PSK_BF16 ? 2 : 4;
    st = check_strides(sh->B, sh->H, sh->n, sh->q_stride_b, sh->q_stride_h, sh->q_stride_n, esz);
    return st != PSK_OK ? st : check_strides(sh->B, sh->Hkv, sh->n, sh->kv_stride_b, sh->kv_stride_h, sh->kv_stride_n, esz);
}
static void plan_parts(WinArgs& a, int tile) {
    a.parts = a.part_rows = a.split_row = 0;
    if (a.sinks == 0 || a.sinks > tile) return;
    const int64_t split = ((int64_t)tile + a.window - 1 + 63) / 64 * 64;               // rows before it see more than the sinks
    if (split >= a.n) return;
    const int64_t base = split / 64, rest = (a.n - split + 63) / 64;                   // steps of 64 rows
    if (rest <= base) return;
    // parts no longer than the other tiles' work, and no more of them than keep the GPU busy
    const int64_t keyheads = (int64_t)a.B * a.Hkv, most = 1024 / keyheads + 1, want = (rest + (base > 8 ? base : 8) - 1) / (base > 8 ? base : 8);
    const int64_t parts = want < most ? want : most;
    a.split_row = (int)split;
    a.part_rows = (int)((rest + parts - 1) / parts * 64);
    a.parts = (int)((a.n - split + a.part_rows - 1) / a.part_rows);
}
WinArgs key_side(const WinArgs& a, int tile) {
    WinArgs k = a;
    k.hs = 1;
    // Places that the GPU has for CTAs, and the least rows of an item that are worth the sum behind it (a step of 64 rows takes the tensor cores
    // 0.8 us, the CUDA cores up to 18; the sum 4 to 10).  8 query heads x 2000 rows on one key head, window 500, us: bf16 61 -> 19 + 7, fp32 846 -> 173 + 8.
    const int64_t items = ((int64_t)a.n + tile - 1) / tile * a.B * a.Hkv, places = tile == 128 ? 148 : 444, least = (tile == 128 ? 24 : 4) * 64;
    const int64_t seen = (int64_t)a.window + tile < a.n ? (int64_t)a.window + tile : a.n;
    if (items < places && a.G > 1 && seen * a.G >= least)
        for (k.hs = 2; k.hs < a.G && (a.G % k.hs != 0 || items * k.hs < places); ++k.hs) {}
    k.Hkv *= k.hs;
    k.G /= k.hs;
    plan_parts(k, tile);
    return k;
}
// Bytes of the sums over query heads and over parts.
static size_t row_sum_bytes(const WinArgs& k) { return k.hs > 1 ? (size_t)k.B * k.Hkv * k.n * 2 * 64 * sizeof(float) : 0; }
static size_t partial_bytes(const WinArgs& k) { return k.parts > 0 ? (size_t)k.B * k.Hkv * (k.parts + 1) * 2 * k.sinks * 64 * sizeof(float) : 0; }
// Bytes of the lists of rows that the tensor-core kernels form again (psk_window_tc.cu); k: null for the forward.
static size_t redo_bytes(const WinArgs& a, const WinArgs* k) {
    // (the forward's 8 entries an item, the query side's 4; one workspace may serve both calls)
    const size_t tiles = ((size_t)a.n + 127) / 128, rows = tiles * a.B * a.H, keys = k == nullptr ? 0 : (tiles + k->parts) * k->B * k->Hkv;
    return (rows > keys ? rows : keys) * 8 * sizeof(uint2);
}
static bool on_tensor_cores(const psk_window_shape* sh) { return sh->dtype == PSK_BF16 && sh->path != PSK_PATH_CUDA_CORES; }
// Device waits are bounded by a second, and some last as long as a tile: 2^25 rows of query heads on one tile of keys take the key side 0.4 s.
static int check_attention(const psk_window_shape* sh) {
    const int st = check_rows(sh);
    if (st != PSK_OK || !on_tensor_cores(sh)) return st;
    const int64_t band = (int64_t)sh->window + 128, rows = sh->sinks > 0 || band > sh->n ? sh->n : band;
    return rows * (sh->H / sh->Hkv) < (int64_t)1 << 25 ? PSK_OK : PSK_ERR_UNSUPPORTED;
}
WinArgs args_of(const psk_window_shape* sh) {
    WinArgs a{};
    a.hs = 1;
    a.B = sh->B; a.H = sh->H; a.Hkv = sh->Hkv; a.G = sh->H / sh->Hkv; a.n = sh->n;
    a.window = sh->window; a.sinks = sh->sinks;
    a.scale = sh->scale; a.c = sh->scale * kLog2e;
    // (an extent of 1 gets a stride that a tensor map takes)
    a.qb = sh->B > 1 ? sh->q_stride_b : 64; a.qh = sh->H > 1 ? sh->q_stride_h : 64; a.qn = sh->n > 1 ? sh->q_stride_n : 64;
    a.kb = sh->B > 1 ? sh->kv_stride_b : 64; a.kh = sh->Hkv > 1 ? sh->kv_stride_h : 64; a.kn = sh->n > 1 ? sh->kv_stride_n : 64;
    return a;
}

}  // namespace win
}  // namespace psk

using namespace psk;
using namespace psk::win;

extern "C" {

size_t psk_window_workspace_bytes(const psk_window_shape* shape, int for_backward) {
    if (check_attention(shape) != PSK_OK) return 0;
    const WinArgs a = args_of(shape);
    if (!for_backward) return kStatusBytes + (shape->dtype == PSK_BF16 ? align_up(redo_bytes(a, nullptr)) : 0);
    size_t sums = 0;                                      // (enough for either path)
    for (int tile = kTile; tile <= 128; tile += 64) {
        const WinArgs k = key_side(a, tile);
        const size_t bytes = align_up(row_sum_bytes(k)) + align_up(partial_bytes(k)) + (tile == 128 && shape->dtype == PSK_BF16 ? align_up(redo_bytes(a, &k)) : 0);
        if (bytes > sums) sums = bytes;
    }
    const size_t rows = align_up((size_t)a.B * a.H * a.n * sizeof(float));
    return kStatusBytes + 2 * rows + (shape->dtype == PSK_BF16 ? 2 * rows : 0) + sums;
}

int psk_window_attn_fwd(const psk_window_shape* shape, const void* Q, const void* K, const void* V, const int32_t* lengths, void* O, float* lse,
                        void* workspace, size_t workspace_bytes, void* stream) {
    const int st = check_attention(shape);
    if (st != PSK_OK) return st;
    if (!Q || !K || !V || !O || !lse) return PSK_ERR_INVALID_ARG;
    for (const void* p : {Q, K, V, (const void*)O})
        if (!aligned16(p)) return PSK_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(lengths)) & 3u) return PSK_ERR_ALIGN;
    if (!workspace || workspace_bytes < psk_window_workspace_bytes(shape, 0) || (reinterpret_cast<uintptr_t>(workspace) % kAlign)) return PSK_ERR_WORKSPACE;
    CountLaunches count;
    cudaStream_t s = (cudaStream_t)stream;
    WinArgs a = args_of(shape);
    a.Q = Q; a.K = K; a.V = V; a.out = O; a.lse = lse; a.lengths = lengths;
    int* status = static_cast<int*>(workspace);
    a.redo = reinterpret_cast<uint2*>(static_cast<char*>(workspace) + kStatusBytes);
    cudaError_t e;
    if (on_tensor_cores(shape)) {
        e = tc_window_fwd(a, status, s);
    } else {
        a.status = status;
        e = shape->dtype == PSK_F32 ? cc_window_fwd<float>(a, s) : cc_window_fwd<bf16>(a, s);
    }
    return e == cudaSuccess ? PSK_OK : PSK_ERR_CUDA;
}

int psk_window_attn_bwd(const psk_window_shape* shape, const void* Q, const void* K, const void* V, const int32_t* lengths, const void* O,
                        const float* lse, const void* dO, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes, void* stream) {
    const int st = check_attention(shape);
    if (st != PSK_OK) return st;
    if (!Q || !K || !V || !O || !lse || !dO || !dQ || !dK || !dV) return PSK_ERR_INVALID_ARG;
    for (const void* p : {Q, K, V, O, dO, (const void*)dQ, (const void*)dK, (const void*)dV})
        if (!aligned16(p)) return PSK_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(lengths)) & 3u) return PSK_ERR_ALIGN;
    if (!workspace || workspace_bytes < psk_window_workspace_bytes(shape, 1) || (reinterpret_cast<uintptr_t>(workspace) % kAlign)) return PSK_ERR_WORKSPACE;
    CountLaunches count;
    cudaStream_t s = (cudaStream_t)stream;
    WinArgs a = args_of(shape);
    a.Q = Q; a.K = K; a.V = V; a.O = O; a.lse_in = lse; a.dO = dO; a.dQ = dQ; a.dK = dK; a.dV = dV; a.lengths = lengths;
    a.stat_l = reinterpret_cast<float*>(static_cast<char*>(workspace) + kStatusBytes);
    a.stat_d = a.stat_l + align_up((size_t)a.B * a.H * a.n * sizeof(float)) / sizeof(float);
    WinArgs k = key_side(a, on_tensor_cores(shape) ? 128 : kTile);
    a.stat_r = a.stat_d + align_up((size_t)a.B * a.H * a.n * sizeof(float)) / sizeof(float);
    k.rows = a.stat_r + (shape->dtype == PSK_BF16 ? 2 * align_up((size_t)a.B * a.H * a.n * sizeof(float)) / sizeof(float) : 0);
    k.partial = k.rows + align_up(row_sum_bytes(k)) / sizeof(float);
    // (first the query side's, then the key side's)
    a.redo = k.redo = reinterpret_cast<uint2*>(k.partial + align_up(partial_bytes(k)) / sizeof(float));
    int* status = static_cast<int*>(workspace);
    cudaError_t e;
    if (on_tensor_cores(shape)) {
        e = tc_window_bwd(a, k, status, s);
    } else {
        a.status = status;
        e = shape->dtype == PSK_F32 ? cc_window_bwd<float>(a, k, s) : cc_window_bwd<bf16>(a, k, s);
    }
    if (e == cudaSuccess) e = key_sums(k, shape->dtype == PSK_BF16, s);
    return e == cudaSuccess ? PSK_OK : PSK_ERR_CUDA;
}

}  // extern "C"

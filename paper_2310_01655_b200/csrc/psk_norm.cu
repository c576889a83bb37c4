// Layer normalisation of rows (Section 2.1: queries and keys come normalised to the attention), forward and backward.
//   y = (x - mean) rstd gain + bias,   mean = sum(x) / C,   rstd = 1 / sqrt(sum((x - mean)^2) / C + eps)
//   with a = dy gain,  xhat = (x - mean) rstd:
//   dx = rstd (a - sum(a) / C - xhat sum(a xhat) / C),   dgain = sum over rows of dy xhat,   dbias = sum over rows of dy
// Bound: memory.  A row is read once and stays in registers; the backward forms mean and rstd again from the x that it
// reads anyway, so that nothing but x is kept from the forward (for rows of 64 in bf16 two stored floats would be 6 % of
// the forward's bytes).  All sums in fp32, the variance from the deviations (two passes over registers).
// A row belongs to G = 4 to 32 lanes of a warp, to 2 or 4 warps, or to a CTA; which, by how many accesses it has (a lane keeps up to 32
// values: a row's own work, its addresses, its sums over lanes, its root, is shared by few lanes).  The next row is on its way while one is
// worked on.  Values are handled in packed pairs: with scalar arithmetic the issue slots bound the backward of rows of 64 (1.57 M rows: 236 us).
// Rows whose address or stride is not a multiple of 16 bytes are read by two values, and those of odd length, stride or start value by value.
#include "fast_div.cuh"
#include "packed.cuh"
#include "psk_internal.cuh"

#include <math.h>

namespace psk {
namespace {

typedef __nv_bfloat16 bf16;
constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32, kNormMaxCols = 8192;

struct NormArgs {
    const void *x, *y;                // y: dY (backward only)
    void* z;                          // Y or dX
    const float *gain, *bias;
    float *dgain, *dbias, *partial;   // partial [gridDim.x][2][cols], unless there is one CTA
    uint32_t rows;
    int cols;
    float eps, over_cols;
    FastDiv n1, n2;
    int64_t xs[3], ys[3], zs[3];
};

__device__ __forceinline__ int64_t row_offset(const NormArgs& a, const int64_t (&s)[3], uint32_t r) {
    const uint32_t q = a.n2.div(r), i2 = r - q * a.n2.d, i0 = a.n1.div(q), i1 = q - i0 * a.n1.d;
    return (int64_t)i0 * s[0] + (int64_t)i1 * s[1] + (int64_t)i2 * s[2];
}

// Values are handled in pairs (f2), or one by one where rows are read so.
template <int V> struct Word { typedef f2 type; };
template <> struct Word<1> { typedef float type; };
__device__ __forceinline__ f2 vadd(f2 a, f2 b) { return add2(a, b); }
__device__ __forceinline__ f2 vmul(f2 a, f2 b) { return mul2(a, b); }
__device__ __forceinline__ f2 vfma(f2 a, f2 b, f2 c) { return fma2(a, b, c); }
__device__ __forceinline__ float vsum(f2 a) { return lo2(a) + hi2(a); }
__device__ __forceinline__ float vat(f2 a, int i) { return i ? hi2(a) : lo2(a); }
__device__ __forceinline__ void vset(f2& a, float v) { a = pack2(v, v); }
__device__ __forceinline__ void vload(f2& a, const float* p) { a = pack2(p[0], p[1]); }
__device__ __forceinline__ float vadd(float a, float b) { return a + b; }
__device__ __forceinline__ float vmul(float a, float b) { return a * b; }
__device__ __forceinline__ float vfma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float vsum(float a) { return a; }
__device__ __forceinline__ float vat(float a, int) { return a; }
__device__ __forceinline__ void vset(float& a, float v) { a = v; }
__device__ __forceinline__ void vload(float& a, const float* p) { a = p[0]; }

// V values at p: 16 bytes, two values, or one
template <typename T, int V> struct Pack;
template <> struct Pack<float, 4> {
    float4 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(f2* f) const { f[0] = pack2(v.x, v.y); f[1] = pack2(v.z, v.w); }
    __device__ __forceinline__ static void store(float* p, const f2* f) { *reinterpret_cast<float4*>(p) = make_float4(lo2(f[0]), hi2(f[0]), lo2(f[1]), hi2(f[1])); }
};
template <> struct Pack<bf16, 8> {
    uint4 v;
    __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(f2* f) const {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack2(u[i] << 16, u[i] & 0xffff0000u);
    }
    __device__ __forceinline__ static void store(bf16* p, const f2* f) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(hi2(f[i])), "f"(lo2(f[i])));
        *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <> struct Pack<float, 2> {
    float2 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float2*>(p); }
    __device__ __forceinline__ void zero() { v = make_float2(0.f, 0.f); }
    __device__ __forceinline__ void get(f2* f) const { f[0] = pack2(v.x, v.y); }
    __device__ __forceinline__ static void store(float* p, const f2* f) { *reinterpret_cast<float2*>(p) = make_float2(lo2(f[0]), hi2(f[0])); }
};
template <> struct Pack<bf16, 2> {
    uint32_t v;
    __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint32_t*>(p); }
    __device__ __forceinline__ void zero() { v = 0u; }
    __device__ __forceinline__ void get(f2* f) const { f[0] = pack2(v << 16, v & 0xffff0000u); }
    __device__ __forceinline__ static void store(bf16* p, const f2* f) {
        uint32_t u;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi2(f[0])), "f"(lo2(f[0])));
        *reinterpret_cast<uint32_t*>(p) = u;
    }
};
template <typename T> struct Pack<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void zero() { stf(&v, 0.f); }
    __device__ __forceinline__ void get(float* f) const { f[0] = ldf(&v); }
    __device__ __forceinline__ static void store(T* p, const float* f) { stf(p, f[0]); }
};

// Sums of N values over the lanes of a row, in every lane.  `red`: shared memory for the rows of several warps, which meet at a
// barrier of their own; callers alternate between two of them, so that one barrier per sum is enough.
template <int G, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float (*red)[kNormWarps]) {
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    if constexpr (G > 32) {
        const int group = threadIdx.x / G;
        if (threadIdx.x % 32 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i][threadIdx.x / 32] = s[i];
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(G) : "memory");
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = 0.f;
#pragma unroll
            for (int w = 0; w < G / 32; ++w) s[i] += red[i][group * (G / 32) + w];
        }
    }
}

// s / cols: the product with the reciprocal, and its remainder (a row of one repeated value has that value as its mean)
__device__ __forceinline__ float over_cols(const NormArgs& a, float s) {
    const float m = s * a.over_cols;
    return fmaf(fmaf(-m, (float)a.cols, s), a.over_cols, m);
}

// A row's lanes, and what they hold: accesses l, l + G, ... of V values each, as kPer words each.
template <typename T, int V, int NV, int G> struct RowMap {
    static constexpr int kRowsPerCta = kNormThreads / G, kPer = (V + 1) / 2, kPairs = kPer * NV, kValues = V * NV;
    // rows in flight per lane, as registers allow.  Backward: beside two sums (and the gain) of every column, two rows of x and dy fit 128 registers
    // up to 8 values a lane, and up to 16 where these are bf16 in pairs (16 384 rows in fp32, us with two / one: 4096 columns 243 / 174, 3002 236 / 172).
    static constexpr int kFwdRows = kValues <= 16 ? 4 : 3, kBwdRows = kValues <= (sizeof(T) == 2 && V > 1 ? 16 : 8) ? 2 : 1;
};
// a parameter's values at the lane's columns (1 or 0 where there is none)
template <int V> __device__ __forceinline__ void load_param(typename Word<V>::type* f, const float* p, int vec, bool in, float none) {
#pragma unroll
    for (int i = 0; i < (V + 1) / 2; ++i) {
        if (in && p != nullptr) vload(f[i], p + vec * V + 2 * i);
        else vset(f[i], none);
    }
}
template <typename T, int V, int NV, int G>
__device__ __forceinline__ void load_row(Pack<T, V> (&x)[NV], const NormArgs& a, const void* base, const int64_t (&strides)[3], uint64_t r, int l, int nvec) {
    const T* row = (const T*)base + (r < a.rows ? row_offset(a, strides, (uint32_t)r) : 0);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int vec = l + k * G;
        if (r < a.rows && vec < nvec) x[k].load(row + vec * V); else x[k].zero();
    }
}

template <typename T, int V, int NV, int G>
__global__ void __launch_bounds__(kNormThreads)
norm_fwd_kernel(const __grid_constant__ NormArgs a) {
    using M = RowMap<T, V, NV, G>;
    typedef typename Word<V>::type W;
    constexpr int P = M::kPer, D = M::kFwdRows;
    constexpr bool kKeep = M::kValues <= 24;              // gain and bias in registers, or read again for every row (from L1)
    __shared__ float red[2][1][kNormWarps];
    pdl_sync();
    const int l = threadIdx.x % G, group = threadIdx.x / G, nvec = a.cols / V;
    W gain[kKeep ? M::kPairs : 1], bias[kKeep ? M::kPairs : 1];
    if constexpr (kKeep)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int vec = l + k * G;
            load_param<V>(gain + k * P, a.gain, vec, vec < nvec, 1.f);
            load_param<V>(bias + k * P, a.bias, vec, vec < nvec, 0.f);
        }
    const uint64_t step = (uint64_t)gridDim.x * M::kRowsPerCta;
    Pack<T, V> next[D][NV];
    uint64_t r = (uint64_t)blockIdx.x * M::kRowsPerCta + group;
#pragma unroll
    for (int d = 0; d < D; ++d) load_row<T, V, NV, G>(next[d], a, a.x, a.xs, r + d * step, l, nvec);
    // (the number of rounds is the same for all lanes of a CTA: rows beyond the last are computed as zeros and not stored)
    for (uint64_t r0 = (uint64_t)blockIdx.x * M::kRowsPerCta; r0 < a.rows; r0 += D * step) {
#pragma unroll
      for (int d = 0; d < D; ++d, r += step) {
        if (r0 + d * step >= a.rows) break;
        W f[M::kPairs];
#pragma unroll
        for (int k = 0; k < NV; ++k) next[d][k].get(f + k * P);
        load_row<T, V, NV, G>(next[d], a, a.x, a.xs, r + D * step, l, nvec);
        W s2, q2;
        vset(s2, 0.f);
        vset(q2, 0.f);
#pragma unroll
        for (int i = 0; i < M::kPairs; ++i) s2 = vadd(s2, f[i]);
        float s[1] = {vsum(s2)};
        row_sums<G>(s, red[0]);
        const float mean = over_cols(a, s[0]);
        W mean2;
        vset(mean2, -mean);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (l + k * G < nvec)
#pragma unroll
                for (int i = 0; i < P; ++i) { W& v = f[k * P + i]; v = vadd(v, mean2); q2 = vfma(v, v, q2); }
        float q[1] = {vsum(q2)};
        row_sums<G>(q, red[1]);
        const float rstd = rsqrtf(fmaf(q[0], a.over_cols, a.eps));
        W rstd2;
        vset(rstd2, rstd);
        if (r < a.rows) {
            T* row = (T*)a.z + row_offset(a, a.zs, (uint32_t)r);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int vec = l + k * G;
                if (vec >= nvec) continue;
                W g[P], b[P];
                if constexpr (kKeep) {
#pragma unroll
                    for (int i = 0; i < P; ++i) { g[i] = gain[k * P + i]; b[i] = bias[k * P + i]; }
                } else {
                    load_param<V>(g, a.gain, vec, true, 1.f);
                    load_param<V>(b, a.bias, vec, true, 0.f);
                }
#pragma unroll
                for (int i = 0; i < P; ++i) f[k * P + i] = vfma(vmul(f[k * P + i], rstd2), g[i], b[i]);
                Pack<T, V>::store(row + vec * V, f + k * P);
            }
        }
      }
    }
}

template <typename T, int V, int NV, int G>
__global__ void __launch_bounds__(kNormThreads, RowMap<T, V, NV, G>::kValues <= 16 ? 2 : 1)
norm_bwd_kernel(const __grid_constant__ NormArgs a) {
    using M = RowMap<T, V, NV, G>;
    typedef typename Word<V>::type W;
    constexpr int P = M::kPer, D = M::kBwdRows;
    // the gain in registers, or read again for every row (from L1): where that takes wide accesses and they are short (4096 columns in fp32 174 / 160,
    // 3002, by twos, 172 / 202)
    constexpr bool kKeep = M::kValues <= (sizeof(T) == 4 && V == 4 ? 8 : 16);
    __shared__ float red1[1][kNormWarps], red2[3][kNormWarps];
    extern __shared__ float sums[];                                       // [2][cols]
    pdl_sync();
    const int l = threadIdx.x % G, group = threadIdx.x / G, nvec = a.cols / V;
    W dg[M::kPairs], db[M::kPairs], gain[kKeep ? M::kPairs : 1];
#pragma unroll
    for (int i = 0; i < M::kPairs; ++i) { vset(dg[i], 0.f); vset(db[i], 0.f); }
    if constexpr (kKeep)
#pragma unroll
        for (int k = 0; k < NV; ++k) load_param<V>(gain + k * P, a.gain, l + k * G, l + k * G < nvec, 1.f);
    const uint64_t step = (uint64_t)gridDim.x * M::kRowsPerCta;
    Pack<T, V> nx[D][NV], ny[D][NV];
    uint64_t r = (uint64_t)blockIdx.x * M::kRowsPerCta + group;
#pragma unroll
    for (int d = 0; d < D; ++d) {
        load_row<T, V, NV, G>(nx[d], a, a.x, a.xs, r + d * step, l, nvec);
        load_row<T, V, NV, G>(ny[d], a, a.y, a.ys, r + d * step, l, nvec);
    }
    for (uint64_t r0 = (uint64_t)blockIdx.x * M::kRowsPerCta; r0 < a.rows; r0 += D * step) {
#pragma unroll
      for (int d = 0; d < D; ++d, r += step) {
        if (r0 + d * step >= a.rows) break;
        Pack<T, V> x[NV], y[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) { x[k] = nx[d][k]; y[k] = ny[d][k]; }
        load_row<T, V, NV, G>(nx[d], a, a.x, a.xs, r + D * step, l, nvec);
        load_row<T, V, NV, G>(ny[d], a, a.y, a.ys, r + D * step, l, nvec);
        W s2;
        vset(s2, 0.f);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            W f[P];
            x[k].get(f);
#pragma unroll
            for (int i = 0; i < P; ++i) s2 = vadd(s2, f[i]);
        }
        float s[1] = {vsum(s2)};
        row_sums<G>(s, red1);
        const float mean = over_cols(a, s[0]);
        W mean2;
        vset(mean2, -mean);
        // sums of the squared deviations, of g = dy gain, and of g times the deviation
        W t2[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) vset(t2[i], 0.f);
        auto gained = [&](W (&g)[P], const W (&d)[P], int k) {
            if constexpr (kKeep) {
#pragma unroll
                for (int i = 0; i < P; ++i) g[i] = vmul(d[i], gain[k * P + i]);
            } else {
                load_param<V>(g, a.gain, l + k * G, true, 1.f);
#pragma unroll
                for (int i = 0; i < P; ++i) g[i] = vmul(d[i], g[i]);
            }
        };
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (l + k * G >= nvec) continue;
            W f[P], d[P], g[P];
            x[k].get(f);
            y[k].get(d);
            gained(g, d, k);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const W dev = vadd(f[i], mean2);
                t2[0] = vfma(dev, dev, t2[0]);
                t2[1] = vadd(t2[1], g[i]);
                t2[2] = vfma(g[i], dev, t2[2]);
            }
        }
        float t[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) t[i] = vsum(t2[i]);
        row_sums<G>(t, red2);
        const float rstd = rsqrtf(fmaf(t[0], a.over_cols, a.eps));
        // dx = rstd g - rstd sum(g) / C - xhat rstd (rstd sum(g dev) / C), xhat = dev rstd.  (In this order: for spreads beyond 1e13 or
        // below 1e-13 the cube of rstd is not a normal number any more, while xhat and its product with g are near one.)
        const float k1 = -rstd * t[1] * a.over_cols, k2 = -rstd * (rstd * (t[2] * a.over_cols));
        W rstd2, k12, k22;
        vset(rstd2, rstd);
        vset(k12, k1);
        vset(k22, k2);
        if (r < a.rows) {
            T* row = (T*)a.z + row_offset(a, a.zs, (uint32_t)r);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int vec = l + k * G;
                if (vec >= nvec) continue;
                W f[P], d[P], g[P];
                x[k].get(f);
                y[k].get(d);
                gained(g, d, k);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const W dev = vadd(f[i], mean2), xhat = vmul(dev, rstd2);
                    // (by twos, 16 values or more, xhat does not fit the registers as well: 16 384 rows of 3002 in bf16, 97 us so, 136 as the others; rows of 1002 136, 131)
                    dg[k * P + i] = V == 2 && M::kValues > 8 ? vfma(vmul(d[i], rstd2), dev, dg[k * P + i]) : vfma(d[i], xhat, dg[k * P + i]);
                    db[k * P + i] = vadd(db[k * P + i], d[i]);
                    f[i] = vfma(xhat, k22, vfma(g[i], rstd2, k12));
                }
                Pack<T, V>::store(row + vec * V, f);
            }
        }
      }
    }
    if (a.dgain == nullptr && a.dbias == nullptr) return;
    // this CTA's sums over its rows: the rows side by side in a warp first, then warp after warp (a fixed order)
#pragma unroll
    for (int o = G; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < M::kPairs; ++i) {
            dg[i] = vadd(dg[i], __shfl_xor_sync(0xffffffffu, dg[i], o));
            db[i] = vadd(db[i], __shfl_xor_sync(0xffffffffu, db[i], o));
        }
    constexpr int kTurns = G > 32 ? kNormThreads / G : kNormWarps;
    const int turn = G > 32 ? group : (int)threadIdx.x / 32;
    const bool first_rows = G > 32 || threadIdx.x % 32 < G;
    for (int w = 0; w < kTurns; ++w) {
        if (first_rows && turn == w)
#pragma unroll
            for (int i = 0; i < M::kValues; ++i) {
                const int vec = l + i / V * G, c = vec * V + i % V, at = i / V * P + i % V / 2;
                if (vec < nvec) {
                    sums[c] = (w > 0 ? sums[c] : 0.f) + vat(dg[at], i % V % 2);
                    sums[a.cols + c] = (w > 0 ? sums[a.cols + c] : 0.f) + vat(db[at], i % V % 2);
                }
            }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < a.cols; c += kNormThreads) {
        if (gridDim.x > 1) {
            float* out = a.partial + (size_t)blockIdx.x * 2 * a.cols;
            out[c] = sums[c];
            out[a.cols + c] = sums[a.cols + c];
        } else {
            if (a.dgain != nullptr) a.dgain[c] = sums[c];
            if (a.dbias != nullptr) a.dbias[c] = sums[a.cols + c];
        }
    }
}

// Sums of the CTAs' partial sums: 32 columns by 32 rows of threads.
constexpr int kSumRows = 32;
__global__ void __launch_bounds__(32 * kSumRows)
norm_sum_kernel(const float* __restrict__ partial, int parts, int cols, float* __restrict__ dgain, float* __restrict__ dbias) {
    __shared__ float s[kSumRows][33];
    pdl_sync();
    const int tx = threadIdx.x % 32, ty = threadIdx.x / 32, c = blockIdx.x * 32 + tx;
    float t = 0.f;
    if (c < 2 * cols)
#pragma unroll 4
        for (int p = ty; p < parts; p += kSumRows) t += partial[(size_t)p * 2 * cols + c];
    s[ty][tx] = t;
    __syncthreads();
    // (transposed: a warp sums one column)
    float u = s[tx][ty];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    const int oc = blockIdx.x * 32 + ty;
    if (tx == 0 && oc < 2 * cols) {
        if (oc < cols) { if (dgain != nullptr) dgain[oc] = u; }
        else if (dbias != nullptr) dbias[oc - cols] = u;
    }
}

// ---- host ----

constexpr int kNormMaxCtas = 148 * 2;           // (with rows in flight two per SM are enough, and fewer sums are left to add up)

// extents and strides in the order of X's strides, so that neighbouring rows are read together
struct Order { int32_t n[3]; int idx[3]; };
Order order_of(const psk_norm_shape* sh) {
    Order o{{sh->n0, sh->n1, sh->n2}, {0, 1, 2}};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (sh->xs[o.idx[j]] < sh->xs[o.idx[j + 1]] && o.n[j + 1] > 1) {
                const int t = o.idx[j]; o.idx[j] = o.idx[j + 1]; o.idx[j + 1] = t;
                const int32_t m = o.n[j]; o.n[j] = o.n[j + 1]; o.n[j + 1] = m;
            }
    return o;
}

// Rows that are written must not overlap: every extent steps over what lies inside it.
bool rows_apart(const int32_t (&n)[3], const int64_t* s, int cols) {
    int64_t end = cols;
    bool used[3] = {false, false, false};
    for (int k = 0; k < 3; ++k) {
        int at = -1;
        for (int i = 0; i < 3; ++i)
            if (!used[i] && n[i] > 1 && (at < 0 || s[i] < s[at])) at = i;
        if (at < 0) return true;
        used[at] = true;
        if (s[at] < end || s[at] > ((int64_t)1 << 44) / (n[at] - 1)) return false;      // (no memory is that large)
        end = s[at] * (n[at] - 1) + end;
    }
    return true;
}

int check_shape(const psk_norm_shape* sh, bool backward) {
    if (sh == nullptr) return PSK_ERR_INVALID_ARG;
    if (sh->dtype != PSK_F32 && sh->dtype != PSK_BF16) return PSK_ERR_INVALID_ARG;
    if (!(sh->eps >= 0.f) || isinf(sh->eps)) return PSK_ERR_INVALID_ARG;
    if (sh->n0 <= 0 || sh->n1 <= 0 || sh->n2 <= 0 || sh->cols <= 0) return PSK_ERR_SHAPE;
    if (sh->cols > kNormMaxCols) return PSK_ERR_UNSUPPORTED;
    if ((int64_t)sh->n0 * sh->n1 >= (int64_t)1 << 31 || (int64_t)sh->n0 * sh->n1 * sh->n2 >= (int64_t)1 << 31) return PSK_ERR_SHAPE;
    const int32_t n[3] = {sh->n0, sh->n1, sh->n2};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (sh->xs[i] < 0 || (backward && sh->ys[i] < 0))) return PSK_ERR_SHAPE;
    return rows_apart(n, backward ? sh->zs : sh->ys, sh->cols) ? PSK_OK : PSK_ERR_SHAPE;
}

template <typename M>
int grid_of(const NormArgs& a) {
    const uint64_t want = ((uint64_t)a.rows + M::kRowsPerCta - 1) / M::kRowsPerCta;
    return (int)(want < (uint64_t)kNormMaxCtas ? want : (uint64_t)kNormMaxCtas);
}
template <typename T, int V, int NV, int G>
cudaError_t launch_fwd(const NormArgs& a, cudaStream_t s) {
    prof_begin("norm_fwd_kernel", s);
    launch_pdl(norm_fwd_kernel<T, V, NV, G>, dim3(grid_of<RowMap<T, V, NV, G>>(a)), dim3(kNormThreads), 0, s, a);
    prof_end(s);
    return cudaGetLastError();
}
template <typename T, int V, int NV, int G>
cudaError_t launch(const NormArgs& a, bool backward, cudaStream_t s) {
    if (!backward) return launch_fwd<T, V, NV, G>(a, s);
    const int grid = grid_of<RowMap<T, V, NV, G>>(a);
    const bool params = a.dgain != nullptr || a.dbias != nullptr;
    const size_t smem = params ? 2 * (size_t)a.cols * sizeof(float) : 0;
    cudaError_t e = cudaFuncSetAttribute(norm_bwd_kernel<T, V, NV, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kNormMaxCols * (int)sizeof(float));
    if (e != cudaSuccess) return e;
    prof_begin("norm_bwd_kernel", s);
    launch_pdl(norm_bwd_kernel<T, V, NV, G>, dim3(grid), dim3(kNormThreads), smem, s, a);
    prof_end(s);
    if (params && grid > 1) {
        prof_begin("norm_sum_kernel", s);
        launch_pdl(norm_sum_kernel, dim3((2 * a.cols + 31) / 32), dim3(32 * kSumRows), 0, s, (const float*)a.partial, grid, a.cols, a.dgain, a.dbias);
        prof_end(s);
    }
    return cudaGetLastError();
}

template <typename T>
cudaError_t dispatch(const NormArgs& a, int width, bool backward, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int nvec = a.cols / width;
    if (width == 2) {                     // (65 536 rows of 1002, bf16, us by twos / one by one: forward 87 / 101, backward 134 / 154; 16 384 of 3002: 68 / 115, 111 / 410)
        if (nvec <= 32) return launch<T, 2, 1, 32>(a, backward, s);
        if (nvec <= 128) return launch<T, 2, 4, 32>(a, backward, s);
        if (nvec <= 256) return launch<T, 2, 4, 64>(a, backward, s);
        if (nvec <= 512) return launch<T, 2, 4, 128>(a, backward, s);
        if (nvec <= 1024) return launch<T, 2, 4, 256>(a, backward, s);
        if (nvec <= 2048) return launch<T, 2, 8, 256>(a, backward, s);
        return launch<T, 2, 16, 256>(a, backward, s);
    }
    if (width == 1) {
        if (nvec <= 32) return launch<T, 1, 1, 32>(a, backward, s);
        if (nvec <= 128) return launch<T, 1, 4, 32>(a, backward, s);
        if (nvec <= 256) return launch<T, 1, 8, 32>(a, backward, s);
        if (nvec <= 512) return launch<T, 1, 8, 64>(a, backward, s);
        if (nvec <= 1024) return launch<T, 1, 8, 128>(a, backward, s);
        if (nvec <= 2048) return launch<T, 1, 8, 256>(a, backward, s);
        if (nvec <= 4096) return launch<T, 1, 16, 256>(a, backward, s);
        return launch<T, 1, 32, 256>(a, backward, s);
    }
    if (nvec <= 8) return launch<T, V, 2, 4>(a, backward, s);
    if (nvec <= 16) return launch<T, V, 2, 8>(a, backward, s);
    if (nvec <= 32) return launch<T, V, 2, 16>(a, backward, s);
    if (nvec <= 64) return launch<T, V, 2, 32>(a, backward, s);
    // (the forward has the registers for more values in a lane; 65 536 rows of 768, us with 32 / 64 lanes to a row: forward 44 / 57, backward 179 / 85)
    if (!backward && nvec <= 96) return launch_fwd<T, V, 3, 32>(a, s);
    if (nvec <= 128) return launch<T, V, 2, 64>(a, backward, s);
    if (nvec <= 256) return launch<T, V, 2, 128>(a, backward, s);
    if (nvec <= 512) return launch<T, V, 2, 256>(a, backward, s);
    if (nvec <= 1024) return launch<T, V, 4, 256>(a, backward, s);
    if constexpr (V == 4) return launch<T, V, 8, 256>(a, backward, s);
    return cudaErrorInvalidValue;
}

int run(const psk_norm_shape* sh, NormArgs& a, bool backward, cudaStream_t s) {
    const Order o = order_of(sh);
    a.rows = (uint32_t)sh->n0 * (uint32_t)sh->n1 * (uint32_t)sh->n2;
    a.cols = sh->cols;
    a.eps = sh->eps;
    a.over_cols = 1.f / (float)sh->cols;
    a.n1.set((uint32_t)o.n[1]);
    a.n2.set((uint32_t)o.n[2]);
    // values that every row can be read by at once: 16 bytes' worth, two, or one
    const int esz = sh->dtype == PSK_F32 ? 4 : 2;
    int width = 16 / esz;
    auto whole = [&](int64_t values, uintptr_t bytes) {
        while (width > 1 && (values % width != 0 || bytes % (uintptr_t)(width * esz) != 0)) width = width > 2 ? 2 : 1;
    };
    whole(sh->cols, 0);
    for (const void* p : {a.x, a.y, (const void*)a.z}) whole(0, reinterpret_cast<uintptr_t>(p));
    const int64_t* in = sh->xs;
    for (int i = 0; i < 3; ++i) {
        const int k = o.idx[i];
        a.xs[i] = in[k];
        a.ys[i] = backward ? sh->ys[k] : 0;
        a.zs[i] = backward ? sh->zs[k] : sh->ys[k];
        if (o.n[i] > 1)
            for (int64_t v : {a.xs[i], a.ys[i], a.zs[i]}) whole(v, 0);
    }
    const cudaError_t e = sh->dtype == PSK_F32 ? dispatch<float>(a, width, backward, s) : dispatch<bf16>(a, width, backward, s);
    return e == cudaSuccess ? PSK_OK : PSK_ERR_CUDA;
}

}  // namespace
}  // namespace psk

using namespace psk;

extern "C" {

size_t psk_layer_norm_workspace_bytes(const psk_norm_shape* shape) {
    if (check_shape(shape, true) != PSK_OK) return 0;
    // partial sums of the most CTAs that a call has (a CTA has a row at least)
    const uint64_t rows = (uint64_t)shape->n0 * shape->n1 * shape->n2;
    const uint64_t ctas = rows < (uint64_t)kNormMaxCtas ? rows : (uint64_t)kNormMaxCtas;
    return align_up((size_t)ctas * 2 * shape->cols * sizeof(float));
}

int psk_layer_norm_fwd(const psk_norm_shape* shape, const void* X, const float* gain, const float* bias, void* Y, void* stream) {
    const int st = check_shape(shape, false);
    if (st != PSK_OK) return st;
    if (!X || !Y) return PSK_ERR_INVALID_ARG;
    CountLaunches count;
    NormArgs a{};
    a.x = X; a.z = Y; a.gain = gain; a.bias = bias;
    return run(shape, a, false, (cudaStream_t)stream);
}

int psk_layer_norm_bwd(const psk_norm_shape* shape, const void* X, const float* gain, const void* dY, void* dX, float* dgain, float* dbias,
                       void* workspace, size_t workspace_bytes, void* stream) {
    const int st = check_shape(shape, true);
    if (st != PSK_OK) return st;
    if (!X || !dY || !dX) return PSK_ERR_INVALID_ARG;
    if (dgain != nullptr || dbias != nullptr) {
        if (!workspace || workspace_bytes < psk_layer_norm_workspace_bytes(shape) || (reinterpret_cast<uintptr_t>(workspace) & 15u)) return PSK_ERR_WORKSPACE;
    }
    CountLaunches count;
    NormArgs a{};
    a.x = X; a.y = dY; a.z = dX; a.gain = gain; a.dgain = dgain; a.dbias = dbias;
    a.partial = static_cast<float*>(workspace);
    return run(shape, a, true, (cudaStream_t)stream);
}

}  // extern "C"

// Sliding-window softmax attention: what its kernels share.
//   row i of a sequence of length L (i < L) sees key j <=> j <= i and (i - j < window or j < sinks)
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp(s_ij),  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
//   D_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - D_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
// Scores are kept times log2(e), so that exponentials are powers of two.
#pragma once

#include "psk_internal.cuh"

namespace psk {
namespace win {

typedef __nv_bfloat16 bf16;

struct WinArgs {
    const void *Q, *K, *V, *O, *dO;
    void *out, *dQ, *dK, *dV;         // `out`: O of the forward
    const float* lse_in;
    float* lse;
    float *stat_l, *stat_d;           // [B,H,n] scratch: -lse log2(e) and -D, written by the query side, read by the key side
    float* stat_r;                    // [2][B,H,n] scratch of the query side on the tensor cores: sums of ds over a third of a row's steps
    const int32_t* lengths;           // [B] or null
    int* status;                      // the call's status word; its first kernel clears it (CUDA-core kernels)
    int B, H, Hkv, G, n, window, sinks;
    float scale, c;                   // c = scale log2(e)
    int64_t qb, qh, qn, kb, kh, kn;   // element strides of the query-side and of the key-side tensors
    // Key side: the tile with the sinks is seen by every row of its sequence, any other by a window's.  Where that makes it much longer, the rows
    // from `split_row` on are left to `parts` items of `part_rows` rows each, and the sinks' gradients are added up from
    // `partial` [B Hkv][parts + 1][dK, dV][sinks][64] in a fixed order (part 0: the rows before split_row).  parts = 0: nothing of that.
    int parts, part_rows, split_row;
    float* partial;
    // Key side: where key heads and tiles are too few for the GPU, the query heads that share a key head are dealt to `hs` heads that do as
    // if they were key heads of their own (Hkv and G there: times and through hs); their sums are added up from `rows` [B Hkv][dK, dV][n][64].
    int hs;
    float* rows;
    // Tensor-core kernels: rows that are formed again when a CTA has done all else, [item](x [2], key side)[warps of its rows] (redo_* below)
    uint2* redo;
};
__device__ __forceinline__ float* sum_row(const WinArgs& a, int b, int hk, int which, int j) {
    return a.rows + ((((int64_t)b * a.Hkv + hk) * 2 + which) * a.n + j) * 64;
}
__device__ __forceinline__ float* partial_row(const WinArgs& a, int b, int hk, int part, int which, int j) {
    return a.partial + ((((int64_t)b * a.Hkv + hk) * (a.parts + 1) + part) * 2 + which) * a.sinks * 64 + (int64_t)j * 64;
}

__device__ __forceinline__ int length_of(const WinArgs& a, int b) {
    if (a.lengths == nullptr) return a.n;
    const int l = a.lengths[b];
    return l < 0 ? 0 : (l > a.n ? a.n : l);
}
// (i - j and i - window + 1 do not overflow: 0 <= i, j < 2^31, window >= 1)
__device__ __forceinline__ bool sees(int i, int j, int window, int sinks) { return j <= i && (i - j < window || j < sinks); }
// the first key of row i's window
__device__ __forceinline__ int window_start(int i, int window) { return i - window + 1 > 0 ? i - window + 1 : 0; }

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// ---- single rows by one warp, pair by pair ----
// The tiled kernels multiply the weight 0 of a pair that the mask leaves out with the other row's values.  If an infinity or a NaN
// stands there, it comes through as NaN.  So a result row that is not finite, though its own statistics are no NaN, and that shares a tile with
// such a row that it does not see (*_tainted) is formed again here from the pairs that count alone (lane l holds columns 2 l and
// 2 l + 1).  Slow, and only there: eight pairs on their way at a time, and no further than to the pair that makes all of
// the row NaN.  In the tensor-core kernels waits have a limit of a second, and a row over a long sequence takes a warp longer: there such rows
// are only noted, and looked at when nobody in the CTA waits any more.
constexpr int kRedo = 8;
// (p: of an even column, of a row on 16 bytes)
__device__ __forceinline__ float2 ld2(const float* p) { return *reinterpret_cast<const float2*>(p); }
__device__ __forceinline__ float2 ld2(const bf16* p) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
template <typename T> __device__ __forceinline__ void st2(T* p, float2 v) { stf(p, v.x); stf(p + 1, v.y); }
__device__ __forceinline__ float dot2(float2 a, float2 b) { return fmaf(a.x, b.x, a.y * b.y); }
__device__ __forceinline__ bool all_nan(float2 v) { return __all_sync(0xffffffffu, v.x != v.x && v.y != v.y); }
__device__ __forceinline__ void warp_sums(float (&v)[kRedo]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int u = 0; u < kRedo; ++u) v[u] += __shfl_xor_sync(0xffffffffu, v[u], o);
}
// The keys of row i by number: those of the sinks before its window, then its window.
struct RowKeys {
    int lo, first;
    __device__ __forceinline__ RowKeys(int i, int window, int sinks) : lo(window_start(i, window)) { first = sinks < lo ? sinks : lo; }
    __device__ __forceinline__ int count(int i) const { return first + i - lo + 1; }
    __device__ __forceinline__ int at(int t) const { return t < first ? t : lo + t - first; }
};

// Is any value of the rows r0 .. r1 - 1 of A or B not finite?
template <typename T>
__device__ __noinline__ bool rows_tainted(const T* A, const T* B, int64_t stride, int r0, int r1) {
    const int l2 = 2 * (threadIdx.x % 32);
    float zero = 0.f;                                     // (becomes NaN with any infinity or NaN)
#pragma unroll 8
    for (int r = r0; r < r1; ++r) {
        const float2 a = ld2(A + r * stride + l2), b = ld2(B + r * stride + l2);
        zero += a.x * 0.f + a.y * 0.f + b.x * 0.f + b.y * 0.f;
    }
    return __any_sync(0xffffffffu, zero != 0.f);
}
// Query side, row i of a sequence of `len`: keys that it does not see and that tiles of up to 128 rows and keys bring with it.
template <typename T>
__device__ __noinline__ bool row_tainted(const T* K, const T* V, int64_t kn, int i, int window, int sinks, int len) {
    const int lo = window_start(i, window), before = lo > 256 ? lo - 256 : 0, after = len - i > 128 ? i + 128 : len;
    const int64_t tile = ((int64_t)sinks + 127) / 128 * 128;
    return rows_tainted(K, V, kn, before, lo) || rows_tainted(K, V, kn, i + 1, after) || (sinks > 0 && rows_tainted(K, V, kn, sinks, (int)(tile < lo ? tile : lo)));
}

// q, K, V: of row i and of its head
template <typename T>
__device__ __noinline__ float2 redo_out_row(const T* q, const T* K, const T* V, int64_t kn, int i, int window, int sinks, float c) {
    const int l2 = 2 * (threadIdx.x % 32);
    const float2 qv = ld2(q + l2);
    const RowKeys keys(i, window, sinks);
    const int count = keys.count(i);
    float m = neg_inf(), l = 0.f;
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int t = 0; t < count && !all_nan(acc); t += kRedo) {
        float s[kRedo];
        float2 v[kRedo];
#pragma unroll
        for (int u = 0; u < kRedo; ++u) {
            const int64_t at = keys.at(t + u < count ? t + u : t) * kn + l2;
            s[u] = dot2(qv, ld2(K + at));
            v[u] = ld2(V + at);
        }
        warp_sums(s);
        float top = m;                                    // (a NaN score: p is NaN, and so is the row)
#pragma unroll
        for (int u = 0; u < kRedo; ++u) { s[u] *= c; top = t + u < count ? fmaxf(top, s[u]) : top; }
        const float base = top == neg_inf() ? 0.f : top, alpha = exp2_approx(m - base);
        acc.x *= alpha;
        acc.y *= alpha;
        l *= alpha;
        m = top;
#pragma unroll
        for (int u = 0; u < kRedo; ++u) {
            if (t + u >= count) break;
            const float p = exp2_approx(s[u] - base);
            acc.x = fmaf(p, v[u].x, acc.x);
            acc.y = fmaf(p, v[u].y, acc.y);
            l += p;
        }
    }
    return make_float2(acc.x / l, acc.y / l);
}

template <typename T>
__device__ __noinline__ float2 redo_dq_row(const T* q, const T* dO, const T* K, const T* V, int64_t kn, int i, int window, int sinks, float c, float scale,
                                           float2 stat) {
    const int l2 = 2 * (threadIdx.x % 32);
    const float2 qv = ld2(q + l2), dv = ld2(dO + l2);
    const RowKeys keys(i, window, sinks);
    const int count = keys.count(i);
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int t = 0; t < count && !all_nan(acc); t += kRedo) {
        float s[kRedo], d[kRedo];
        float2 k[kRedo];
#pragma unroll
        for (int u = 0; u < kRedo; ++u) {
            const int64_t at = keys.at(t + u < count ? t + u : t) * kn + l2;
            k[u] = ld2(K + at);
            s[u] = dot2(qv, k[u]);
            d[u] = dot2(dv, ld2(V + at));
        }
        warp_sums(s);
        warp_sums(d);
#pragma unroll
        for (int u = 0; u < kRedo; ++u) {
            if (t + u >= count) break;
            const float ds = exp2_approx(fmaf(s[u], c, -stat.x)) * (d[u] - stat.y);
            acc.x = fmaf(ds, k[u].x, acc.x);
            acc.y = fmaf(ds, k[u].y, acc.y);
        }
    }
    return make_float2(acc.x * scale, acc.y * scale);
}

// Key side, key j: query rows that do not see it and that tiles bring with it (keys in tiles of up to 128, rows in steps of up to 64, before `stop`).
template <typename T>
__device__ __noinline__ bool key_tainted(const WinArgs& a, int b, int hk, int j, int len, int stop) {
    const int64_t past = (int64_t)j + a.window;
    const int before = j > 127 ? j - 127 : 0, most = len < stop ? len : stop;
    int r0 = most, r1 = most;                             // behind its window
    if (j >= a.sinks && past < most) {
        r0 = (int)past;
        if (j / 128 * 128 >= a.sinks && most - r0 > 192) r1 = r0 + 192;
        if (r1 - r0 > a.window + 192) return true;        // (more rows than those that count: look at these instead)
    }
    for (int g = 0; g < a.G; ++g) {
        const int h = hk * a.G + g;
        const int64_t at = b * a.qb + h * a.qh;
        if (rows_tainted((const T*)a.Q + at, (const T*)a.dO + at, a.qn, before, j) || rows_tainted((const T*)a.Q + at, (const T*)a.dO + at, a.qn, r0, r1)) return true;
        const float *sl = a.stat_l + ((int64_t)b * a.H + h) * a.n, *sd = a.stat_d + ((int64_t)b * a.H + h) * a.n;
        bool bad = false;
        for (int r = before + (int)(threadIdx.x % 32); r < j; r += 32) bad = bad || !finite(sl[r]) || !finite(sd[r]);
        for (int r = r0 + (int)(threadIdx.x % 32); r < r1; r += 32) bad = bad || !finite(sl[r]) || !finite(sd[r]);
        if (__any_sync(0xffffffffu, bad)) return true;
    }
    return false;
}

// row j of key head hk of sequence b: (dk, dv), from the query rows before `stop`
struct KeyRow { float2 dk, dv; };
template <typename T>
__device__ __noinline__ KeyRow redo_dkv_row(const WinArgs& a, int b, int hk, int j, int len, int stop) {
    const int l2 = 2 * (threadIdx.x % 32);
    const int64_t krow = b * a.kb + hk / a.hs * a.kh + j * a.kn + l2;
    const float2 k = ld2((const T*)a.K + krow), v = ld2((const T*)a.V + krow);
    KeyRow r{make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    const int64_t past = (int64_t)j + a.window;
    const int most = len < stop ? len : stop, end = (j < a.sinks || past > most) ? most : (int)past;
    for (int g = 0; g < a.G; ++g) {
        const int h = hk * a.G + g;
        const T *Q = (const T*)a.Q + b * a.qb + h * a.qh + l2, *dO = (const T*)a.dO + b * a.qb + h * a.qh + l2;
        const float *sl = a.stat_l + ((int64_t)b * a.H + h) * a.n, *sd = a.stat_d + ((int64_t)b * a.H + h) * a.n;
#pragma unroll 1
        for (int i0 = j; i0 < end && !(all_nan(r.dk) && all_nan(r.dv)); i0 += kRedo) {
            float s[kRedo], e[kRedo];
            float2 q[kRedo], d[kRedo];
#pragma unroll
            for (int u = 0; u < kRedo; ++u) {
                const int i = end - i0 > u ? i0 + u : i0;
                q[u] = ld2(Q + i * a.qn);
                d[u] = ld2(dO + i * a.qn);
                s[u] = dot2(q[u], k);
                e[u] = dot2(d[u], v);
            }
            warp_sums(s);
            warp_sums(e);
#pragma unroll
            for (int u = 0; u < kRedo; ++u) {
                if (end - i0 <= u) break;
                const float p = exp2_approx(fmaf(s[u], a.c, sl[i0 + u])), ds = p * (e[u] + sd[i0 + u]) * a.scale;
                r.dv.x = fmaf(p, d[u].x, r.dv.x); r.dv.y = fmaf(p, d[u].y, r.dv.y);
                r.dk.x = fmaf(ds, q[u].x, r.dk.x); r.dk.y = fmaf(ds, q[u].y, r.dk.y);
            }
        }
    }
    return r;
}

// The key tiles (of `tile` keys) that rows row0 .. row1 see any key of: [0, sink_tiles) and [band0, band1].
struct KeyTiles {
    int sink_tiles, band0, band1;
    __device__ __forceinline__ int count() const { return sink_tiles + band1 - band0 + 1; }
    __device__ __forceinline__ int at(int x) const { return x < sink_tiles ? x : band0 + x - sink_tiles; }
};
__device__ __forceinline__ KeyTiles key_tiles(int row0, int row1, int window, int sinks, int tile) {
    KeyTiles k;
    k.band0 = window_start(row0, window) / tile;
    k.band1 = row1 / tile;
    const int s = (int)(((int64_t)sinks + tile - 1) / tile);
    k.sink_tiles = s < k.band0 ? s : k.band0;
    return k;
}
// The last row (exclusive) that sees any of the keys key0 .. key1 of a sequence of `len`: later ones see none.
__device__ __forceinline__ int rows_end(int key0, int key1, int window, int sinks, int len) {
    const int64_t past = (int64_t)key1 + window;
    return (key0 < sinks || past > len) ? len : (int)past;
}

// The work of a key-side item: the keys key0 .. of a head, the query rows from `begin` on and before `stop`, and which part of the sinks' sums
// they make (-1: those are not split).  Items before the tiles' are the parts of the sinks' tile.
struct KeyItem {
    int b, h, key0, len, begin, stop, part;
    __device__ __forceinline__ bool empty() const { return begin >= stop; }
    // one past its last row (not kept: a register of the loop over the rows)
    __device__ __forceinline__ int end(const WinArgs& a, int tile) const {
        const int e = rows_end(key0, (key0 + tile < len ? key0 + tile : len) - 1, a.window, a.sinks, len);
        return e < stop ? e : stop;
    }
};
template <typename D1, typename D2, typename D3>
__device__ __forceinline__ KeyItem key_item(const WinArgs& a, int index, int tile, const D1& by_tiles, const D2& by_heads, const D3& by_parts) {
    KeyItem k;
    const int first = a.parts * a.B * a.Hkv;              // (the parts first: they are the longer ones)
    int bh, q = -1;
    if (index >= first) { bh = by_tiles(index - first); k.key0 = (index - first - bh * ((a.n + tile - 1) / tile)) * tile; }
    else { bh = by_parts(index); q = index - bh * a.parts; k.key0 = 0; }
    k.b = by_heads(bh);
    k.h = bh - k.b * a.Hkv;
    k.len = length_of(a, k.b);
    k.begin = k.key0;
    k.stop = k.len;
    k.part = -1;
    if (a.parts > 0 && k.key0 == 0) {
        if (q < 0) {
            k.stop = k.len < a.split_row ? k.len : a.split_row;
        } else {
            k.begin = a.split_row + q * a.part_rows;
            k.stop = k.len - k.begin < a.part_rows ? k.len : k.begin + a.part_rows;
        }
        k.part = q + 1;
    }
    return k;
}

// host: argument checks and what the kernels take (psk_window.cu)
int check_common(const psk_window_shape* sh);         // all but n and the strides
int check_rows(const psk_window_shape* sh);
WinArgs args_of(const psk_window_shape* sh);
WinArgs key_side(const WinArgs& a, int tile);         // as the key side takes them: with hs, parts, part_rows, split_row
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// tensor cores (psk_window_tc.cu): bf16
cudaError_t tc_window_fwd(const WinArgs& a, int* status, cudaStream_t s);
cudaError_t tc_window_bwd(const WinArgs& a, const WinArgs& k, int* status, cudaStream_t s);      // k: for the key side

}  // namespace win
}  // namespace psk

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
    const int32_t* lengths;           // [B] or null
    int* status;                      // the call's status word; its first kernel clears it
    int B, H, Hkv, G, n, window, sinks;
    float scale, c;                   // c = scale log2(e)
    int64_t qb, qh, qn, kb, kh, kn;   // element strides of the query-side and of the key-side tensors
    // Key side: the tile with the sinks is seen by every row of its sequence, any other by a window's.  Where that makes it much longer, the rows
    // from `split_row` on are left to `parts` items of `part_rows` rows each, and the sinks' gradients are added up from
    // `partial` [B Hkv][parts + 1][dK, dV][sinks][64] in a fixed order (part 0: the rows before split_row).  parts = 0: nothing of that.
    int parts, part_rows, split_row;
    float* partial;
};
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

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---- single rows by one warp, pair by pair ----
// The tiled kernels multiply the weight 0 of a pair that the mask leaves out with the other row's values.  If an infinity or a NaN
// stands there, it comes through as NaN.  So a result row that is not finite is formed again here from
// the pairs that count alone (lane l holds columns 2 l and 2 l + 1).  Slow, and only there.
template <typename T> __device__ __forceinline__ float2 ld2(const T* p) { return make_float2(ldf(p), ldf(p + 1)); }
template <typename T> __device__ __forceinline__ void st2(T* p, float2 v) { stf(p, v.x); stf(p + 1, v.y); }
__device__ __forceinline__ float dot2(float2 a, float2 b) { return warp_sum(fmaf(a.x, b.x, a.y * b.y)); }

template <typename F>
__device__ __forceinline__ void for_keys(int i, int window, int sinks, F&& f) {
    const int lo = window_start(i, window), first = sinks < lo ? sinks : lo;
    for (int j = 0; j < first; ++j) f(j);
    for (int j = lo; j <= i; ++j) f(j);
}

// q, K, V: of row i and of its head; lse: its place, or null
template <typename T>
__device__ __noinline__ float2 redo_out_row(const T* q, const T* K, const T* V, int64_t kn, int i, int window, int sinks, float c, float* lse) {
    const int l2 = 2 * (threadIdx.x % 32);
    const float2 qv = ld2(q + l2);
    float m = neg_inf(), l = 0.f;
    float2 acc = make_float2(0.f, 0.f);
    for_keys(i, window, sinks, [&](int j) {
        const float s = dot2(qv, ld2(K + j * kn + l2)) * c;
        const float m2 = fmaxf(m, s);                     // (a NaN score: p is NaN, and so is the row)
        const float base = m2 == neg_inf() ? 0.f : m2, alpha = exp2_approx(m - base), p = exp2_approx(s - base);
        const float2 v = ld2(V + j * kn + l2);
        acc.x = fmaf(acc.x, alpha, p * v.x);
        acc.y = fmaf(acc.y, alpha, p * v.y);
        l = fmaf(l, alpha, p);
        m = m2;
    });
    if (l2 == 0 && lse != nullptr) *lse = (m + log2f(l)) * kLn2;
    return make_float2(acc.x / l, acc.y / l);
}

template <typename T>
__device__ __noinline__ float2 redo_dq_row(const T* q, const T* dO, const T* K, const T* V, int64_t kn, int i, int window, int sinks, float c, float scale,
                                           float2 stat) {
    const int l2 = 2 * (threadIdx.x % 32);
    const float2 qv = ld2(q + l2), dv = ld2(dO + l2);
    float2 acc = make_float2(0.f, 0.f);
    for_keys(i, window, sinks, [&](int j) {
        const float2 k = ld2(K + j * kn + l2);
        const float p = exp2_approx(fmaf(dot2(qv, k), c, -stat.x));
        const float ds = p * (dot2(dv, ld2(V + j * kn + l2)) - stat.y);
        acc.x = fmaf(ds, k.x, acc.x);
        acc.y = fmaf(ds, k.y, acc.y);
    });
    return make_float2(acc.x * scale, acc.y * scale);
}

// row j of key head hk of sequence b: (dk, dv), from the query rows before `stop`
struct KeyRow { float2 dk, dv; };
template <typename T>
__device__ __noinline__ KeyRow redo_dkv_row(const WinArgs& a, int b, int hk, int j, int len, int stop) {
    const int l2 = 2 * (threadIdx.x % 32);
    const int64_t krow = b * a.kb + hk * a.kh + j * a.kn + l2;
    const float2 k = ld2((const T*)a.K + krow), v = ld2((const T*)a.V + krow);
    KeyRow r{make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    const int64_t past = (int64_t)j + a.window;
    const int most = len < stop ? len : stop, end = (j < a.sinks || past > most) ? most : (int)past;
    for (int g = 0; g < a.G; ++g) {
        const int h = hk * a.G + g;
        for (int i = j; i < end; ++i) {
            const int64_t row = b * a.qb + h * a.qh + i * a.qn + l2;
            const int64_t at = ((int64_t)b * a.H + h) * a.n + i;
            const float2 q = ld2((const T*)a.Q + row), d = ld2((const T*)a.dO + row);
            const float p = exp2_approx(fmaf(dot2(q, k), a.c, a.stat_l[at]));
            const float ds = p * (dot2(d, v) + a.stat_d[at]) * a.scale;
            r.dv.x = fmaf(p, d.x, r.dv.x); r.dv.y = fmaf(p, d.y, r.dv.y);
            r.dk.x = fmaf(ds, q.x, r.dk.x); r.dk.y = fmaf(ds, q.y, r.dk.y);
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
void plan_parts(WinArgs& a, int tile);                // fills parts, part_rows, split_row
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// tensor cores (psk_window_tc.cu): bf16
cudaError_t tc_window_fwd(const WinArgs& a, int* status, cudaStream_t s);
cudaError_t tc_window_bwd(const WinArgs& a, int* status, cudaStream_t s);

}  // namespace win
}  // namespace psk

// Sliding-window softmax attention on the tensor cores: bf16 operands, fp32 accumulation in tensor memory, fp32 softmax.
// Scores, weights and their gradients never leave the SM.  Forward and query side: a CTA has one tile of 128 query rows (thread = row),
// a warp that issues its MMAs and one that issues its loads, and half of an SM's tensor memory, so that two CTAs share an SM: one's
// exponentials run under the other's MMAs, and so do its set-up and its stores.  Key side: one CTA per SM (below).
// With head dimension 64 a 128 x 128 tile costs 512 cycles of MMAs and, with 16 exponentials per cycle and SM, 1024
// cycles of those in the forward: exponentials bound it.
#include "tc_common.cuh"
#include "psk_window.cuh"

namespace psk {
namespace win {
namespace {

using namespace tc;

constexpr int kRowThreads = 128, kTcThreads = kRowThreads + 64;       // + the warp that issues MMAs, the warp that loads
constexpr int kMmaWarp = 4, kLoadWarp = 5;

struct TcPlace { int b, h, row0, len; };
__device__ __forceinline__ TcPlace tc_place(const WinArgs& a, int heads) {
    const int tiles = (a.n + 127) / 128, bh = blockIdx.x / tiles;
    TcPlace p;
    p.b = bh / heads;
    p.h = bh % heads;
    p.row0 = (int)(blockIdx.x % tiles) * 128;
    p.len = length_of(a, p.b);
    return p;
}

// N columns of tensor memory in registers, as values.
template <int N> struct Cols {
    uint32_t u[N / 32][32];
    __device__ __forceinline__ void load(uint32_t taddr) {
#pragma unroll
        for (int q = 0; q < N / 32; ++q) tmem_ld32(taddr + q * 32, u[q]);
    }
    __device__ __forceinline__ float operator[](int j) const { return __uint_as_float(u[j / 32][j % 32]); }
    __device__ __forceinline__ void set(int j, float f) { u[j / 32][j % 32] = __float_as_uint(f); }
};

// 64 bf16 values of a row
__device__ __forceinline__ void zero_row(bf16* p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(p + 8 * i) = make_uint4(0, 0, 0, 0);
}

// The rows r0, r0 + 1, ... below `end` and zeros behind them as a TMA load would leave them, by a whole warp.  For the tile in which
// a sequence ends before the tensor does: what stands behind its end would meet weights of zero, and 0 times an infinity is NaN.
// (Its scores are masked by selection; only operands of products with weights need this.)
template <int ROWS>
__device__ __noinline__ void warp_load_tile(uint8_t* dst, const bf16* src, int64_t stride, int r0, int end) {
#pragma unroll 8
    for (int e = threadIdx.x % 32; e < ROWS * 8; e += 32) {
        const int r = e / 8, chunk = e % 8;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r0 + r < end) u = *reinterpret_cast<const uint4*>(src + (int64_t)(r0 + r) * stride + chunk * 8);
        *reinterpret_cast<uint4*>(dst + swz128_offset(r, chunk)) = u;
    }
    fence_proxy_async_smem();
    __syncwarp();
}

// Which columns of a key tile the row of this thread sees: c <= hi and (c >= lo or c < sk).  `all`: every row of its warp sees all
// (the same for the warp).
struct KeyMask { int hi, lo, sk; bool all; };
__device__ __forceinline__ KeyMask key_mask(int i, int i_first, int k0, int tile, int window, int sinks) {
    KeyMask m;
    m.hi = i - k0;
    m.lo = window_start(i, window) - k0;
    m.sk = sinks - k0;                                    // (k0 < n < 2^31, sinks >= 0)
    m.all = k0 + tile - 1 <= i_first && (window_start(i_first + 31, window) <= k0 || m.sk >= tile);
    return m;
}
__device__ __forceinline__ bool seen(const KeyMask& m, int c) { return c <= m.hi && (c >= m.lo || c < m.sk); }

// ---------------------------------------------------------------------------
// Forward.  Steps of 128 keys: S = Q K^T (tensor memory), p = 2^(c s - m) as bf16 beside it, O += p V.
// The row's reference m follows its running maximum only where that has grown by more than 8 (2^8 fits every type
// here): then O is multiplied in tensor memory, which otherwise stays with the MMAs.
// S is free again as soon as the rows have read it into registers: S of the next step is formed under the exponentials of this one.
// ---------------------------------------------------------------------------
struct Fwd {
    static constexpr int kK = 3, kV = 2;                  // stages of keys and of values
    static constexpr int Q = 0, K = 16384, V = K + kK * 16384, bytes = V + kV * 16384 + 1024;
    static constexpr uint32_t kTmem = 256, cS = 0, cP = 128, cO = 192;
};

__global__ void __launch_bounds__(kTcThreads, 2)
tc_win_fwd_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                  const __grid_constant__ WinArgs a, int* status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align1024(smem_raw);
    __shared__ uint64_t bar_q, bar_k[Fwd::kK], bar_v[Fwd::kV], free_k[Fwd::kK], free_v[Fwd::kV], bar_s, bar_read, bar_p, bar_o;
    __shared__ uint32_t tm_slot;
    const int tid = threadIdx.x, warp = warp_index();
    pdl_sync();
    if (blockIdx.x == 0 && tid == 0) *status = 0;
    const TcPlace pl = tc_place(a, a.H);
    const int row0 = pl.row0, len = pl.len;
    bf16* O = (bf16*)a.out + pl.b * a.qb + pl.h * a.qh;
    float* lse = a.lse + ((int64_t)pl.b * a.H + pl.h) * a.n;
    if (row0 >= len) {                                    // behind the sequence's end
        if (tid < 128 && row0 + tid < a.n) { zero_row(O + (int64_t)(row0 + tid) * a.qn); lse[row0 + tid] = neg_inf(); }
        return;
    }
    if (tid == 0) {
        cta_giveup_init();
        mbar_init(&bar_q, 1);
        for (int i = 0; i < Fwd::kK; ++i) { mbar_init(&bar_k[i], 1); mbar_init(&free_k[i], 1); }
        for (int i = 0; i < Fwd::kV; ++i) { mbar_init(&bar_v[i], 1); mbar_init(&free_v[i], 1); }
        mbar_init(&bar_s, 1); mbar_init(&bar_read, 4); mbar_init(&bar_p, 4); mbar_init(&bar_o, 1);
        mbar_fence_init();
    }
    if (warp == kMmaWarp) { tmem_alloc(&tm_slot, Fwd::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tm_slot;
    const int row1 = row0 + 127 < len ? row0 + 127 : len - 1;
    const KeyTiles kt = key_tiles(row0, row1, a.window, a.sinks, 128);
    const int steps = kt.count();
    const int hk = pl.h / a.G;
    if (warp == kLoadWarp) {
        bool ok = true;
        if (elect_one()) {
            mbar_expect_tx(&bar_q, 16384);
            tma_load_4d(smem + Fwd::Q, &mapQ, 0, row0, pl.h, pl.b, &bar_q);
        }
        const bf16* V = (const bf16*)a.V + pl.b * a.kb + hk * a.kh;
        for (int x = 0; x < steps; ++x) {
            const int k0 = kt.at(x) * 128, sk = x % Fwd::kK, sv = x % Fwd::kV;
            if (x >= Fwd::kK) ok = mbar_spin(&free_k[sk], (x / Fwd::kK - 1) & 1, status, kErrMma);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (elect_one()) {
                mbar_expect_tx(&bar_k[sk], 16384);
                tma_load_4d(smem + Fwd::K + sk * 16384, &mapK, 0, k0, hk, pl.b, &bar_k[sk]);
            }
            if (x >= Fwd::kV) ok = mbar_spin(&free_v[sv], (x / Fwd::kV - 1) & 1, status, kErrMma);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const bool ends = len < a.n && k0 + 128 > len;
            if (ends) warp_load_tile<128>(smem + Fwd::V + sv * 16384, V, a.kn, k0, len);
            if (elect_one()) {
                if (ends) {
                    mbar_arrive(&bar_v[sv]);
                } else {
                    mbar_expect_tx(&bar_v[sv], 16384);
                    tma_load_4d(smem + Fwd::V + sv * 16384, &mapV, 0, k0, hk, pl.b, &bar_v[sv]);
                }
            }
        }
    } else if (warp == kMmaWarp) {
        if (elect_one()) {
            constexpr uint32_t idesc_s = idesc_bf16(128, 128, false, false), idesc_o = idesc_bf16(128, 64, false, true);
            const uint64_t qd = smem_desc(smem_u32(smem + Fwd::Q), 0, 1024, kSwz128);
            const uint64_t kd = smem_desc(smem_u32(smem + Fwd::K), 0, 1024, kSwz128), vd = smem_desc(smem_u32(smem + Fwd::V), 0, 1024, kSwz128);
            bool ok = mbar_spin(&bar_q, 0, status, kErrTma);
            for (int x = 0; x <= steps && ok; ++x) {
                if (x < steps) {
                    const int s = x % Fwd::kK;
                    ok = mbar_spin(&bar_k[s], (x / Fwd::kK) & 1, status, kErrTma);
                    if (x > 0) ok = ok && mbar_spin(&bar_read, (x - 1) & 1, status, kErrMma);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ss(tm + Fwd::cS, desc_off(qd, k * 32), desc_off(kd, s * 16384 + k * 32), idesc_s, k > 0);
                    umma_commit(&bar_s);
                    umma_commit(&free_k[s]);
                }
                if (x > 0) {
                    const int y = x - 1, s = y % Fwd::kV;
                    ok = mbar_spin(&bar_v[s], (y / Fwd::kV) & 1, status, kErrTma);
                    ok = ok && mbar_spin(&bar_p, y & 1, status, kErrMma);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 8; ++k) umma_ts(tm + Fwd::cO, tm + Fwd::cP + k * 8, desc_off(vd, s * 16384 + k * 2048), idesc_o, (y > 0 || k > 0) ? 1u : 0u);
                    umma_commit(&bar_o);
                    umma_commit(&free_v[s]);
                }
            }
        }
    } else {
        const uint32_t lane_tm = tm + ((uint32_t)(warp * 32) << 16);
        const int i = row0 + tid, i_first = row0 + warp * 32;
        const float c = a.c;
        bool ok = true;
        float m = neg_inf(), l = 0.f;
        for (int x = 0; x < steps; ++x) {
            const int k0 = kt.at(x) * 128;
            Cols<128> s;
            ok = mbar_wait(&bar_s, x & 1, status, kErrMma) && ok;
            tc_fence_after();
            s.load(lane_tm + Fwd::cS);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (tid % 32 == 0) mbar_arrive(&bar_read);
            const KeyMask km = key_mask(i, i_first, k0, 128, a.window, a.sinks);
            if (!km.all) {
#pragma unroll
                for (int j = 0; j < 128; ++j) s.set(j, seen(km, j) ? s[j] : neg_inf());
            }
            float t0 = neg_inf(), t1 = neg_inf(), t2 = neg_inf(), t3 = neg_inf();
#pragma unroll
            for (int j = 0; j < 128; j += 8) {
                t0 = fmaxf(t0, fmaxf(s[j], s[j + 1])); t1 = fmaxf(t1, fmaxf(s[j + 2], s[j + 3]));
                t2 = fmaxf(t2, fmaxf(s[j + 4], s[j + 5])); t3 = fmaxf(t3, fmaxf(s[j + 6], s[j + 7]));
            }
            const float top = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3));
            const bool grow = (top - m) * c > 8.f;
            float alpha = 1.f;
            if (grow) { alpha = exp2_approx((m - top) * c); m = top; l *= alpha; }
            const float base = m == neg_inf() ? 0.f : m * c;
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int j = 0; j < 128; j += 2) {
                s.set(j, exp2_approx(fmaf(s[j], c, -base)));
                s.set(j + 1, exp2_approx(fmaf(s[j + 1], c, -base)));
                l0 += s[j];
                l1 += s[j + 1];
            }
            l += l0 + l1;
            if (x > 0) {                                  // the weights of the step before have been used, O is complete up to it
                ok = mbar_wait(&bar_o, (x - 1) & 1, status, kErrMma) && ok;
                tc_fence_after();
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t o[16];
                        tmem_ld16(lane_tm + Fwd::cO + q * 16, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                        tmem_st16(lane_tm + Fwd::cO + q * 16, o);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t pk[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) pk[j] = pack_bf16(s[32 * q + 2 * j], s[32 * q + 2 * j + 1]);
                tmem_st16(lane_tm + Fwd::cP + q * 16, pk);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (tid % 32 == 0) mbar_arrive(&bar_p);
        }
        ok = mbar_wait(&bar_o, (steps - 1) & 1, status, kErrMma) && ok;
        tc_fence_after();
        const float inv = 1.f / l, v = (m * c + log2f(l)) * kLn2;
        bool fine = finite(v);
        uint32_t out[32];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t o[32];
            tmem_ld32(lane_tm + Fwd::cO + q * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                const float f0 = __uint_as_float(o[j]) * inv, f1 = __uint_as_float(o[j + 1]) * inv;
                fine = fine && finite(f0) && finite(f1);
                out[16 * q + j / 2] = pack_bf16(f0, f1);
            }
        }
        if (i < len) {
            if (ok && fine) {
                bf16* row = O + (int64_t)i * a.qn;
#pragma unroll
                for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(row + 8 * q) = make_uint4(out[4 * q], out[4 * q + 1], out[4 * q + 2], out[4 * q + 3]);
                lse[i] = v;
            }
        } else if (i < a.n) {
            zero_row(O + (int64_t)i * a.qn);
            lse[i] = neg_inf();
        }
        unsigned bad = __ballot_sync(0xffffffffu, ok && !fine && i < len);
        while (bad != 0) {
            const int r = i_first + __ffs(bad) - 1;
            bad &= bad - 1;
            const int64_t koff = pl.b * a.kb + hk * a.kh;
            redo_out_row((const bf16*)a.Q + pl.b * a.qb + pl.h * a.qh + (int64_t)r * a.qn, (const bf16*)a.K + koff, (const bf16*)a.V + koff, a.kn, r, a.window,
                         a.sinks, c, O + (int64_t)r * a.qn, lse + r);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) { cta_teardown_warp(); tmem_dealloc(tm, Fwd::kTmem); }
}

// ---------------------------------------------------------------------------
// Backward, query side.  Steps of 64 keys: S = Q K^T and dP = dO V^T into tensor memory, ds = p (dP - D) as bf16 into tensor memory,
// dQ += ds K.  D_i = do_i . o_i is formed here and left for the key side.  Q lies in tensor memory (an A operand from there
// leaves the shared-memory path to B: 32 cycles instead of 48 for a step of K with N = 64), dO in shared memory.
// ---------------------------------------------------------------------------
struct Dq {
    static constexpr int kStages = 5;
    static constexpr int G = 0, KV = 16384, bytes = KV + kStages * 16384 + 1024;
    static constexpr uint32_t kTmem = 256, cQ = 0, cDs = 32, cDq = 64, cS = 128, cDp = 192;
};

__global__ void __launch_bounds__(kTcThreads, 2)
tc_win_dq_kernel(const __grid_constant__ CUtensorMap mapG, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                 const __grid_constant__ WinArgs a, int* status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align1024(smem_raw);
    __shared__ uint64_t bar_g, bar_kv[Dq::kStages], free_kv[Dq::kStages], bar_s, bar_read, bar_ds, bar_dq;
    __shared__ uint32_t tm_slot;
    const int tid = threadIdx.x, warp = warp_index();
    pdl_sync();
    if (blockIdx.x == 0 && tid == 0) *status = 0;
    const TcPlace pl = tc_place(a, a.H);
    const int row0 = pl.row0, len = pl.len;
    const int64_t qoff = pl.b * a.qb + pl.h * a.qh, soff = ((int64_t)pl.b * a.H + pl.h) * a.n;
    bf16* dQ = (bf16*)a.dQ + qoff;
    if (row0 >= len) {
        if (tid < 128 && row0 + tid < a.n) { zero_row(dQ + (int64_t)(row0 + tid) * a.qn); a.D[soff + row0 + tid] = 0.f; }
        return;
    }
    if (tid == 0) {
        cta_giveup_init();
        mbar_init(&bar_g, 1);
        for (int i = 0; i < Dq::kStages; ++i) { mbar_init(&bar_kv[i], 1); mbar_init(&free_kv[i], 1); }
        mbar_init(&bar_s, 1); mbar_init(&bar_read, 4); mbar_init(&bar_ds, 4); mbar_init(&bar_dq, 1);
        mbar_fence_init();
    }
    if (warp == kMmaWarp) { tmem_alloc(&tm_slot, Dq::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tm_slot;
    const int row1 = row0 + 127 < len ? row0 + 127 : len - 1;
    const KeyTiles kt = key_tiles(row0, row1, a.window, a.sinks, 64);
    const int steps = kt.count();
    const int hk = pl.h / a.G;
    const uint32_t lane_tm = tm + ((uint32_t)(warp * 32) << 16);
    const int i = row0 + tid, i_first = row0 + warp * 32;
    float D = 0.f, lse2 = 0.f;
    if (warp == kLoadWarp) {
        bool ok = true;
        if (elect_one()) {
            mbar_expect_tx(&bar_g, 16384);
            tma_load_4d(smem + Dq::G, &mapG, 0, row0, pl.h, pl.b, &bar_g);
        }
        const bf16* K = (const bf16*)a.K + pl.b * a.kb + hk * a.kh;
        for (int x = 0; x < steps; ++x) {
            const int k0 = kt.at(x) * 64, s = x % Dq::kStages;
            if (x >= Dq::kStages) ok = mbar_spin(&free_kv[s], (x / Dq::kStages - 1) & 1, status, kErrMma);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            uint8_t* st = smem + Dq::KV + s * 16384;
            const bool ends = len < a.n && k0 + 64 > len;
            if (ends) warp_load_tile<64>(st, K, a.kn, k0, len);
            if (elect_one()) {
                mbar_expect_tx(&bar_kv[s], ends ? 8192 : 16384);
                if (!ends) tma_load_4d(st, &mapK, 0, k0, hk, pl.b, &bar_kv[s]);
                tma_load_4d(st + 8192, &mapV, 0, k0, hk, pl.b, &bar_kv[s]);
            }
        }
    } else if (warp < kMmaWarp) {
        uint32_t q[32];
        if (i < len) {
            const uint4* qr = reinterpret_cast<const uint4*>((const bf16*)a.Q + qoff + (int64_t)i * a.qn);
            const uint4* gr = reinterpret_cast<const uint4*>((const bf16*)a.dO + qoff + (int64_t)i * a.qn);
            const uint4* orow = reinterpret_cast<const uint4*>((const bf16*)a.O + qoff + (int64_t)i * a.qn);
            lse2 = a.lse_in[soff + i] * kLog2e;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint4 u = qr[k], g = gr[k], o = orow[k];
                q[4 * k] = u.x; q[4 * k + 1] = u.y; q[4 * k + 2] = u.z; q[4 * k + 3] = u.w;
                const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    D = fmaf(__uint_as_float(gw[w] << 16), __uint_as_float(ow[w] << 16), D);
                    D = fmaf(__uint_as_float(gw[w] & 0xffff0000u), __uint_as_float(ow[w] & 0xffff0000u), D);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) q[k] = 0;
        }
        if (i < a.n) a.D[soff + i] = D;
        tmem_st32(lane_tm + Dq::cQ, q);
        tmem_st_wait();
    }
    tc_fence_before();
    if (warp != kLoadWarp) asm volatile("bar.sync 1, 160;" ::: "memory");      // Q is in place (the loads are on their way)
    tc_fence_after();
    if (warp == kMmaWarp) {
        if (elect_one()) {
            constexpr uint32_t idesc_s = idesc_bf16(128, 64, false, false), idesc_o = idesc_bf16(128, 64, false, true);
            const uint64_t gd = smem_desc(smem_u32(smem + Dq::G), 0, 1024, kSwz128), kvd = smem_desc(smem_u32(smem + Dq::KV), 0, 1024, kSwz128);
            bool ok = mbar_spin(&bar_g, 0, status, kErrTma);
            for (int x = 0; x <= steps && ok; ++x) {
                if (x < steps) {
                    const int s = x % Dq::kStages;
                    ok = mbar_spin(&bar_kv[s], (x / Dq::kStages) & 1, status, kErrTma);
                    if (x > 0) ok = ok && mbar_spin(&bar_read, (x - 1) & 1, status, kErrMma);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ts(tm + Dq::cS, tm + Dq::cQ + k * 8, desc_off(kvd, s * 16384 + k * 32), idesc_s, k > 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ss(tm + Dq::cDp, desc_off(gd, k * 32), desc_off(kvd, s * 16384 + 8192 + k * 32), idesc_s, k > 0);
                    umma_commit(&bar_s);
                }
                if (x > 0) {
                    const int y = x - 1, s = y % Dq::kStages;
                    ok = mbar_spin(&bar_ds, y & 1, status, kErrMma);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ts(tm + Dq::cDq, tm + Dq::cDs + k * 8, desc_off(kvd, s * 16384 + k * 2048), idesc_o, (y > 0 || k > 0) ? 1u : 0u);
                    umma_commit(&free_kv[s]);
                    umma_commit(&bar_dq);
                }
            }
        }
    } else if (warp < kMmaWarp) {
        const float c = a.c;
        bool ok = true;
        for (int x = 0; x < steps; ++x) {
            const int k0 = kt.at(x) * 64;
            Cols<64> s, d;
            ok = mbar_wait(&bar_s, x & 1, status, kErrMma) && ok;
            tc_fence_after();
            s.load(lane_tm + Dq::cS);
            d.load(lane_tm + Dq::cDp);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (tid % 32 == 0) mbar_arrive(&bar_read);
#pragma unroll
            for (int j = 0; j < 64; ++j) s.set(j, exp2_approx(fmaf(s[j], c, -lse2)) * (d[j] - D));
            const KeyMask km = key_mask(i, i_first, k0, 64, a.window, a.sinks);
            if (!km.all) {
#pragma unroll
                for (int j = 0; j < 64; ++j) s.set(j, seen(km, j) ? s[j] : 0.f);
            }
            uint32_t pk[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) pk[j] = pack_bf16(s[2 * j], s[2 * j + 1]);
            if (x > 0) {
                ok = mbar_wait(&bar_dq, (x - 1) & 1, status, kErrMma) && ok;
                tc_fence_after();
            }
            tmem_st32(lane_tm + Dq::cDs, pk);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (tid % 32 == 0) mbar_arrive(&bar_ds);
        }
        ok = mbar_wait(&bar_dq, (steps - 1) & 1, status, kErrMma) && ok;
        tc_fence_after();
        bool fine = true;
        uint32_t out[32];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t o[32];
            tmem_ld32(lane_tm + Dq::cDq + q * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                const float f0 = __uint_as_float(o[j]) * a.scale, f1 = __uint_as_float(o[j + 1]) * a.scale;
                fine = fine && finite(f0) && finite(f1);
                out[16 * q + j / 2] = pack_bf16(f0, f1);
            }
        }
        if (i < len) {
            if (ok && fine) {
                bf16* row = dQ + (int64_t)i * a.qn;
#pragma unroll
                for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(row + 8 * q) = make_uint4(out[4 * q], out[4 * q + 1], out[4 * q + 2], out[4 * q + 3]);
            }
        } else if (i < a.n) {
            zero_row(dQ + (int64_t)i * a.qn);
        }
        unsigned bad = __ballot_sync(0xffffffffu, ok && !fine && i < len);
        while (bad != 0) {
            const int src = __ffs(bad) - 1, r = i_first + src;
            bad &= bad - 1;
            const int64_t at = (int64_t)r * a.qn, koff = pl.b * a.kb + hk * a.kh;
            redo_dq_row((const bf16*)a.Q + qoff + at, (const bf16*)a.dO + qoff + at, (const bf16*)a.K + koff, (const bf16*)a.V + koff, a.kn, r, a.window, a.sinks, c,
                        a.scale, a.lse_in[soff + r], __shfl_sync(0xffffffffu, D, src), dQ + at);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) { cta_teardown_warp(); tmem_dealloc(tm, Dq::kTmem); }
}

// ---------------------------------------------------------------------------
// Backward, key side: one tile of 128 keys (thread = key), steps of 64 query rows of every query head that shares the key head:
// S^T = K Q^T, dP^T = V dO^T, p^T and ds^T as bf16 operands, dV += p^T dO, dK += ds^T Q.  Four MMAs of 128 cycles a step
// bound it, as long as the next scores are formed while the rows work: that takes two buffers of scores and operands of their
// own for p and ds, all of an SM's tensor memory.  Two warpgroups take the steps in turn.
// ---------------------------------------------------------------------------
struct Dkv {
    static constexpr int kStages = 8, kThreads = 2 * kRowThreads + 64, kMma = 8, kLoad = 9;
    static constexpr int QG = 0, bytes = kStages * 16384 + 1024;
    static constexpr uint32_t kTmem = 512, cK = 0, cV = 32, cDk = 64, cDv = 128, cP = 192, cDs = 224, cS = 256;      // cS + 128 buffer: S, dP
};

__global__ void __launch_bounds__(Dkv::kThreads, 1)
tc_win_dkv_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapG, const __grid_constant__ WinArgs a, int* status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align1024(smem_raw);
    __shared__ __align__(16) float s_lse[Dkv::kStages][64], s_D[Dkv::kStages][64];
    __shared__ int s_bad[128];
    __shared__ uint64_t bar_qg[Dkv::kStages], free_qg[Dkv::kStages], bar_s[2], bar_read[2], bar_done[2], bar_ds;
    __shared__ uint32_t tm_slot;
    const int tid = threadIdx.x, warp = warp_index();
    pdl_sync();
    const TcPlace pl = tc_place(a, a.Hkv);
    const int key0 = pl.row0, len = pl.len;
    const int64_t koff = pl.b * a.kb + pl.h * a.kh;
    bf16 *dK = (bf16*)a.dK + koff, *dV = (bf16*)a.dV + koff;
    if (key0 >= len) {
        if (tid < 256 && key0 + tid % 128 < a.n) zero_row((tid < 128 ? dK : dV) + (int64_t)(key0 + tid % 128) * a.kn);
        return;
    }
    if (tid == 0) {
        cta_giveup_init();
        for (int i = 0; i < Dkv::kStages; ++i) { mbar_init(&bar_qg[i], 1); mbar_init(&free_qg[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_s[i], 1); mbar_init(&bar_read[i], 4); mbar_init(&bar_done[i], 1); }
        mbar_init(&bar_ds, 4);
        mbar_fence_init();
    }
    if (tid < 128) s_bad[tid] = 0;
    if (warp == Dkv::kMma) { tmem_alloc(&tm_slot, Dkv::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tm_slot;
    const int key1 = key0 + 127 < len ? key0 + 127 : len - 1;
    const int q_end = rows_end(key0, key1, a.window, a.sinks, len);
    const int tiles = (q_end - key0 + 63) / 64, steps = tiles * a.G;
    const int group = warp / 4, row = tid % 128, j = key0 + row;
    const uint32_t lane_tm = tm + ((uint32_t)(warp % 4 * 32) << 16);
    if (warp < Dkv::kMma) {                               // K's rows by the first warpgroup, V's by the second
        uint32_t r[32];
        if (j < len) {
            const uint4* p = reinterpret_cast<const uint4*>((const bf16*)(group == 0 ? a.K : a.V) + koff + (int64_t)j * a.kn);
#pragma unroll
            for (int k = 0; k < 8; ++k) { const uint4 u = p[k]; r[4 * k] = u.x; r[4 * k + 1] = u.y; r[4 * k + 2] = u.z; r[4 * k + 3] = u.w; }
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) r[k] = 0;
        }
        tmem_st32(lane_tm + (group == 0 ? Dkv::cK : Dkv::cV), r);
        tmem_st_wait();
    }
    tc_fence_before();
    if (warp != Dkv::kLoad) asm volatile("bar.sync 1, 288;" ::: "memory");     // K and V are in place (the loads start)
    tc_fence_after();
    if (warp == Dkv::kLoad) {
        const int lane = tid % 32;
        bool ok = true;
        for (int x = 0; x < steps; ++x) {
            const int h = pl.h * a.G + x / tiles, i0 = key0 + x % tiles * 64, s = x % Dkv::kStages;
            if (x >= Dkv::kStages) ok = mbar_spin(&free_qg[s], (x / Dkv::kStages - 1) & 1, status, kErrMma);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const int64_t soff = ((int64_t)pl.b * a.H + h) * a.n;
#pragma unroll
            for (int e = lane; e < 64; e += 32) {
                const bool in = i0 + e < len;
                s_lse[s][e] = in ? a.lse_in[soff + i0 + e] * kLog2e : 0.f;
                s_D[s][e] = in ? a.D[soff + i0 + e] : 0.f;
            }
            const bool ends = len < a.n && i0 + 64 > len;
            if (ends) {
                const int64_t off = pl.b * a.qb + h * a.qh;
                warp_load_tile<64>(smem + s * 16384, (const bf16*)a.Q + off, a.qn, i0, len);
                warp_load_tile<64>(smem + s * 16384 + 8192, (const bf16*)a.dO + off, a.qn, i0, len);
            }
            __syncwarp();
            if (elect_one()) {
                if (ends) {
                    mbar_arrive(&bar_qg[s]);
                } else {
                    mbar_expect_tx(&bar_qg[s], 16384);
                    tma_load_4d(smem + s * 16384, &mapQ, 0, i0, h, pl.b, &bar_qg[s]);
                    tma_load_4d(smem + s * 16384 + 8192, &mapG, 0, i0, h, pl.b, &bar_qg[s]);
                }
            }
        }
    } else if (warp == Dkv::kMma) {
        if (elect_one()) {
            constexpr uint32_t idesc_s = idesc_bf16(128, 64, false, false), idesc_o = idesc_bf16(128, 64, false, true);
            const uint64_t qd = smem_desc(smem_u32(smem), 0, 1024, kSwz128);
            bool ok = true;
            // scores of step x two steps ahead of its products
            for (int x = 0; x < steps + 2 && ok; ++x) {
                if (x < steps) {
                    const int s = x % Dkv::kStages, buf = x & 1;
                    ok = mbar_spin(&bar_qg[s], (x / Dkv::kStages) & 1, status, kErrTma);
                    if (x >= 2) ok = ok && mbar_spin(&bar_read[buf], (x / 2 - 1) & 1, status, kErrMma);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ts(tm + Dkv::cS + buf * 128, tm + Dkv::cK + k * 8, desc_off(qd, s * 16384 + k * 32), idesc_s, k > 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ts(tm + Dkv::cS + buf * 128 + 64, tm + Dkv::cV + k * 8, desc_off(qd, s * 16384 + 8192 + k * 32), idesc_s, k > 0);
                    umma_commit(&bar_s[buf]);
                }
                if (x >= 2) {
                    const int y = x - 2, s = y % Dkv::kStages;
                    ok = mbar_spin(&bar_ds, y & 1, status, kErrMma);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ts(tm + Dkv::cDv, tm + Dkv::cP + k * 8, desc_off(qd, s * 16384 + 8192 + k * 2048), idesc_o, (y > 0 || k > 0) ? 1u : 0u);
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_ts(tm + Dkv::cDk, tm + Dkv::cDs + k * 8, desc_off(qd, s * 16384 + k * 2048), idesc_o, (y > 0 || k > 0) ? 1u : 0u);
                    umma_commit(&free_qg[s]);
                    umma_commit(&bar_done[y & 1]);
                }
            }
        }
    } else {
        const float c = a.c;
        bool ok = true;
        for (int x = group; x < steps; x += 2) {
            const int i0 = key0 + x % tiles * 64, st = x % Dkv::kStages;
            Cols<64> s, d;
            ok = mbar_wait(&bar_qg[st], (x / Dkv::kStages) & 1, status, kErrTma) && ok;     // (the rows' statistics)
            ok = mbar_wait(&bar_s[group], (x / 2) & 1, status, kErrMma) && ok;
            tc_fence_after();
            s.load(lane_tm + Dkv::cS + group * 128);
            d.load(lane_tm + Dkv::cS + group * 128 + 64);
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (tid % 32 == 0) mbar_arrive(&bar_read[group]);
#pragma unroll
            for (int e = 0; e < 64; e += 4) {
                const float4 L = *reinterpret_cast<const float4*>(&s_lse[st][e]), D = *reinterpret_cast<const float4*>(&s_D[st][e]);
                const float lv[4] = {L.x, L.y, L.z, L.w}, dv[4] = {D.x, D.y, D.z, D.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    s.set(e + k, exp2_approx(fmaf(s[e + k], c, -lv[k])));
                    d.set(e + k, s[e + k] * (d[e + k] - dv[k]));
                }
            }
            // query rows i0 + e, lo <= e <= hi, see this key
            const int lo = j - i0;
            const int64_t past = (int64_t)j + a.window;
            const int hi = ((j < a.sinks || past > len) ? len : (int)past) - 1 - i0;
            const int w0 = key0 + warp % 4 * 32;          // (the same for the warp:) all of them see all of its keys
            const bool all = w0 + 31 <= i0 && i0 + 63 < len && (i0 + 63 - w0 < a.window || w0 + 31 < a.sinks);
            if (!all) {
#pragma unroll
                for (int e = 0; e < 64; ++e) {
                    const bool v = e >= lo && e <= hi;
                    s.set(e, v ? s[e] : 0.f);
                    d.set(e, v ? d[e] : 0.f);
                }
            }
            uint32_t pk[32], dk[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) { pk[e] = pack_bf16(s[2 * e], s[2 * e + 1]); dk[e] = pack_bf16(d[2 * e], d[2 * e + 1]); }
            if (x > 0) {                                  // the products of the step before have read theirs
                ok = mbar_wait(&bar_done[(x - 1) & 1], ((x - 1) / 2) & 1, status, kErrMma) && ok;
                tc_fence_after();
            }
            tmem_st32(lane_tm + Dkv::cP, pk);
            tmem_st32(lane_tm + Dkv::cDs, dk);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (tid % 32 == 0) mbar_arrive(&bar_ds);
        }
        // (A barrier's parity tells two phases apart.  Each warpgroup waits on one of the two barriers, phase after phase; the
        // phase before the one waited for here has been seen, on it or by way of a later step's.)
        ok = mbar_wait(&bar_done[(steps - 1) & 1], ((steps - 1) / 2) & 1, status, kErrMma) && ok;
        tc_fence_after();
        // the first warpgroup has dK, the second dV
        const float f = group == 0 ? a.scale : 1.f;
        bool fine = true;
        uint32_t out[32];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t o[32];
            tmem_ld32(lane_tm + (group == 0 ? Dkv::cDk : Dkv::cDv) + q * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
                const float f0 = __uint_as_float(o[e]) * f, f1 = __uint_as_float(o[e + 1]) * f;
                fine = fine && finite(f0) && finite(f1);
                out[16 * q + e / 2] = pack_bf16(f0, f1);
            }
        }
        if (j < len && !fine) s_bad[row] = 1;
        asm volatile("bar.sync 2, 256;" ::: "memory");
        bf16* dst = (group == 0 ? dK : dV) + (int64_t)j * a.kn;
        if (j < len) {
            if (ok && !s_bad[row]) {
#pragma unroll
                for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(dst + 8 * q) = make_uint4(out[4 * q], out[4 * q + 1], out[4 * q + 2], out[4 * q + 3]);
            }
        } else if (j < a.n) {
            zero_row(dst);
        }
        if (!cta_gave_up())
            for (int r = warp; r < 128; r += 8)
                if (s_bad[r]) redo_dkv_row<bf16>(a, pl.b, pl.h, key0 + r, len);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == Dkv::kMma) { cta_teardown_warp(); tmem_dealloc(tm, Dkv::kTmem); }
}

}  // namespace

cudaError_t tc_window_fwd(const WinArgs& a, int* status, cudaStream_t s) {
    CUtensorMap mQ, mK, mV;
    if (!tc_map_rows(&mQ, a.Q, a.B, a.H, a.n, a.qb, a.qh, a.qn) || !tc_map_rows(&mK, a.K, a.B, a.Hkv, a.n, a.kb, a.kh, a.kn) ||
        !tc_map_rows(&mV, a.V, a.B, a.Hkv, a.n, a.kb, a.kh, a.kn))
        return cudaErrorInvalidValue;
    PSK_TRY(set_smem(tc_win_fwd_kernel, Fwd::bytes));
    const unsigned tiles = (unsigned)((a.n + 127) / 128);
    prof_begin("tc_win_fwd_kernel", s);
    launch_pdl(tc_win_fwd_kernel, dim3(tiles * a.B * a.H), dim3(kTcThreads), Fwd::bytes, s, mQ, mK, mV, a, status);
    prof_end(s);
    return cudaGetLastError();
}

cudaError_t tc_window_bwd(const WinArgs& a, int* status, cudaStream_t s) {
    CUtensorMap mQ, mG, mG64, mK, mV;
    if (!tc_map_rows(&mQ, a.Q, a.B, a.H, a.n, a.qb, a.qh, a.qn, 64) || !tc_map_rows(&mG, a.dO, a.B, a.H, a.n, a.qb, a.qh, a.qn) ||
        !tc_map_rows(&mG64, a.dO, a.B, a.H, a.n, a.qb, a.qh, a.qn, 64) || !tc_map_rows(&mK, a.K, a.B, a.Hkv, a.n, a.kb, a.kh, a.kn, 64) ||
        !tc_map_rows(&mV, a.V, a.B, a.Hkv, a.n, a.kb, a.kh, a.kn, 64))
        return cudaErrorInvalidValue;
    PSK_TRY(set_smem(tc_win_dq_kernel, Dq::bytes));
    PSK_TRY(set_smem(tc_win_dkv_kernel, Dkv::bytes));
    const unsigned tiles = (unsigned)((a.n + 127) / 128);
    prof_begin("tc_win_dq_kernel", s);
    launch_pdl(tc_win_dq_kernel, dim3(tiles * a.B * a.H), dim3(kTcThreads), Dq::bytes, s, mG, mK, mV, a, status);
    prof_end(s);
    prof_begin("tc_win_dkv_kernel", s);
    launch_pdl(tc_win_dkv_kernel, dim3(tiles * a.B * a.Hkv), dim3(Dkv::kThreads), Dkv::bytes, s, mQ, mG64, a, status);
    prof_end(s);
    return cudaGetLastError();
}

}  // namespace win
}  // namespace psk

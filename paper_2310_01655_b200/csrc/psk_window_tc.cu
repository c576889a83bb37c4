// Sliding-window softmax attention on the tensor cores: bf16 operands, fp32 accumulation in tensor memory, fp32 softmax.
// Scores, weights and their gradients never leave the SM.  Warps have one task each: one issues the loads (TMA), one the MMAs, the
// others hold rows in their threads.  Items of work (a tile of 128 rows of one head) follow one another in a CTA that
// stays: while an item's last exponentials are formed and its result is stored, the next one's operands are loaded
// and its first scores formed.  Which item comes next the hardware says (cluster launch control: a CTA takes over
// one of those that have not been started), so that items of different length even out.
// With head dimension 64 a 128 x 128 tile holds the tensor pipe 512 cycles in the forward and 1270 on either
// side of the backward (operands read from shared memory: 48 cycles for M = 128, N = 64, K = 16, where 16 would do), and the exponential
// unit (16 per cycle and SM) 1024 cycles in each.  It takes 1830, 2600 and 2850: what bounds it is the way from scores to
// rows and back to the next products, under which too few other steps lie.  192 heads x 8192 rows, window 512: 412, 586 and 641 us,
// 480, 510 and 620 TFLOP/s of the pairs that count.
#include "fast_div.cuh"
#include "packed.cuh"
#include "tc_common.cuh"
#include "psk_window.cuh"

namespace psk {
namespace win {
namespace {

using namespace tc;

constexpr int kRows = 128;

// ---------------------------------------------------------------------------
// Items
// ---------------------------------------------------------------------------
struct Item { int b, h, row0, len; };
struct ItemMap { FastDiv tiles, heads, parts; };
__device__ __forceinline__ Item item_of(const WinArgs& a, const ItemMap& m, int index) {
    const int bh = m.tiles.div(index);
    Item p;
    p.b = m.heads.div(bh);
    p.h = bh - p.b * m.heads.d;
    p.row0 = (index - bh * m.tiles.d) * kRows;
    p.len = length_of(a, p.b);
    return p;
}

// The items of a CTA: its own index first, then, where there are more items than places (`takes`), those that it takes over.  The answer behind the it-th item is asked for by the
// loading warp while that item is worked on, and read by every warp.
struct Sched {
    ulonglong2 answer[2];
    uint64_t full[2], taken[2];
};
__device__ __forceinline__ void sched_init(Sched& s, int warps) {
    for (int i = 0; i < 2; ++i) { mbar_init(&s.full[i], 1); mbar_init(&s.taken[i], warps); }
}
// may the place of the it-th answer be written again?
__device__ __forceinline__ bool sched_free(Sched& s, int it, int* status) { return it < 2 || mbar_wait(&s.taken[it & 1], (it / 2 - 1) & 1, status, kErrMma); }
__device__ __forceinline__ void sched_ask(Sched& s, int it, bool takes) {
    if (!takes) return;
    mbar_expect_tx(&s.full[it & 1], 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                 ::"r"(smem_u32(&s.answer[it & 1])), "r"(smem_u32(&s.full[it & 1])) : "memory");
}
// The index of the item behind the it-th; -1: there is none, or a wait gave up.  Followed by sched_taken() from one lane of the warp.
__device__ __forceinline__ int sched_next(Sched& s, int it, bool takes, int* status) {
    if (!takes || !mbar_wait(&s.full[it & 1], (it / 2) & 1, status, kErrTma)) return -1;
    uint64_t lo, hi;
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(lo), "=l"(hi) : "r"(smem_u32(&s.answer[it & 1])) : "memory");
    uint32_t got, index;
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
                 "mov.b128 r, {%2, %3};\n\t"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
                 : "=r"(got), "=r"(index) : "l"(lo), "l"(hi));
    fence_proxy_async_smem();                             // (read before it is written again by the other proxy)
    return got ? (int)index : -1;
}
__device__ __forceinline__ void sched_taken(Sched& s, int it) { mbar_arrive(&s.taken[it & 1]); }

// ---------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------

// N columns of tensor memory in registers, as values.
template <int N> struct Cols {
    uint32_t u[N];
    __device__ __forceinline__ void load(uint32_t taddr) {
        if constexpr (N == 32) tmem_ld32(taddr, u);
        else tmem_ld16(taddr, u);
    }
    __device__ __forceinline__ float operator[](int j) const { return __uint_as_float(u[j]); }
    __device__ __forceinline__ void set(int j, float f) { u[j] = __float_as_uint(f); }
    __device__ __forceinline__ f2 pair(int j) const { return pack2(u[j], u[j + 1]); }       // j even
};

// Named barriers among some of a CTA's threads; the second says whether any of them brought a true value.
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ bool bar_any(int id, int threads, bool v) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, %2, %3, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(r) : "r"((uint32_t)v), "r"(id), "r"(threads) : "memory");
    return r != 0;
}

// Zeros into the rows row0 .. row0 + 127 below n, by THREADS threads.
template <int THREADS>
__device__ __forceinline__ void zero_tile(bf16* p, int64_t stride, int row0, int n, int t) {
#pragma unroll
    for (int k = 0; k < kRows * 8 / THREADS; ++k) {
        const int r = row0 + k * (THREADS / 8) + t / 8;
        if (r < n) *reinterpret_cast<uint4*>(p + (int64_t)r * stride + t % 8 * 8) = make_uint4(0, 0, 0, 0);
    }
}

// Half a row of 64 values (times f, SECOND: plus another's times f1; as bf16; zeros if !live) into a staged tile; true if all of them are finite.
template <bool SECOND = false>
__device__ __forceinline__ bool stage_half(uint8_t* st, int row, int half, uint32_t taddr, float f, bool live, uint32_t taddr1 = 0, float f1 = 0.f) {
    f2 zero = 0;                                          // (becomes NaN with any infinity or NaN)
    const f2 ff = pack2(f, f), ff1 = pack2(f1, f1);
    Cols<32> o, o1;
    o.load(taddr + half * 32);
    if constexpr (SECOND) o1.load(taddr1 + half * 32);
    tmem_ld_wait();
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        f2 v = mul2(o.pair(j), ff);
        if constexpr (SECOND) v = fma2(o1.pair(j), ff1, v);
        zero = fma2(v, 0ull, zero);
        w[j / 2] = live ? pack_bf16(lo2(v), hi2(v)) : 0u;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(st + swz128_offset(row, 4 * half + k)) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    return finite(lo2(zero) + hi2(zero));
}
__device__ __forceinline__ bool stage_row(uint8_t* st, int row, uint32_t taddr, float f, bool live) {
    const bool a = stage_half(st, row, 0, taddr, f, live), b = stage_half(st, row, 1, taddr, f, live);
    return a && b;
}
__device__ __forceinline__ bool stage_row(uint8_t* st, int row, uint32_t taddr, float f, bool live, uint32_t taddr1, float f1) {
    const bool a = stage_half<true>(st, row, 0, taddr, f, live, taddr1, f1), b = stage_half<true>(st, row, 1, taddr, f, live, taddr1, f1);
    return a && b;
}
// A row of 64 values times f into memory as fp32 (where `live`), for sums over parts.
__device__ __forceinline__ void store_partial(float* dst, uint32_t taddr, float f, bool live) {
#pragma unroll 1
    for (int q = 0; q < 64; q += 16) {
        Cols<16> o;
        o.load(taddr + q);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            if (live) *reinterpret_cast<float4*>(dst + q + j) = make_float4(o[j] * f, o[j + 1] * f, o[j + 2] * f, o[j + 3] * f);
    }
}

// Rows to be formed again (psk_window.cuh): a warp's list of items, through memory.  An entry: which of the warp's 32 rows, and the code of the
// item noted before it.
constexpr uint32_t kNoItem = 0xffffffffu;
__device__ __forceinline__ void redo_note(uint2* entry, uint32_t code, unsigned rows, uint32_t& last) {
    if (rows != 0 && threadIdx.x % 32 == 0) { *entry = make_uint2(rows, last); last = code; }
}
// f(code, row) for each, by the whole warp, when the CTA's tiles have arrived in memory
template <typename Entry, typename F>
__device__ __forceinline__ void redo_noted(uint32_t last, const Entry& entry, const F& f) {
#pragma unroll 1
    for (uint32_t code = last; code != kNoItem;) {
        const uint2 e = *entry(code);
#pragma unroll 1
        for (unsigned rows = e.x; rows != 0; rows &= rows - 1) f(code, __ffs(rows) - 1);
        code = e.y;
    }
}

// The rows r0, r0 + 1, ... below `end` and zeros behind them as a TMA load would leave them, by a whole warp.  For the tile in which
// a sequence ends before the tensor does: what stands behind its end would meet weights of zero, and 0 times an infinity is NaN.
// (Scores are masked by selection: the forward's keys do not need this.)
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

// Masks, 32 columns at a time: one bit per column and row.  For most of these chunks all rows of a warp see everything or nothing; those need
// no mask or no exponentials at all (of a window of 512 in steps of 64, one chunk in ten is crossed by an edge).
__device__ __forceinline__ uint32_t bits_below(int k) { return k >= 32 ? 0xffffffffu : (k <= 0 ? 0u : (1u << k) - 1u); }
enum Seen { kNone, kSome, kAll };
__device__ __forceinline__ Seen seen_by_warp(uint32_t w) {
    return __reduce_and_sync(0xffffffffu, w) == 0xffffffffu ? kAll : (__reduce_or_sync(0xffffffffu, w) != 0u ? kSome : kNone);
}
// Columns of a key tile that a query row sees: c <= hi and (c >= lo or c < sk).
struct KeyMask {
    int hi, lo, sk;
    __device__ __forceinline__ uint32_t word(int q) const { return bits_below(hi + 1 - 32 * q) & (~bits_below(lo - 32 * q) | bits_below(sk - 32 * q)); }
};
__device__ __forceinline__ KeyMask key_mask(int i, int k0, int window, int sinks) {
    return KeyMask{i - k0, window_start(i, window) - k0, sinks - k0};                  // (0 <= k0 < n < 2^31, sinks >= 0)
}
// Do the 32 rows from i_first on see all of the keys k0 .. k0 + tile - 1?
__device__ __forceinline__ bool sees_all(int i_first, int k0, int tile, int window, int sinks) {
    return k0 + tile - 1 <= i_first && (window_start(i_first + 31, window) <= k0 || sinks - k0 >= tile);
}
template <int N>
__device__ __forceinline__ void mask_scores(Cols<N>& s, uint32_t w) {
#pragma unroll
    for (int j = 0; j < N; ++j) s.set(j, (w & (1u << j)) ? s[j] : neg_inf());
}
__device__ __forceinline__ void store_zeros(uint32_t taddr) {
    const uint32_t z[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    tmem_st16(taddr, z);
}
// 2^x of a pair
__device__ __forceinline__ f2 exp2_pair(f2 x) { return pack2(exp2_approx(lo2(x)), exp2_approx(hi2(x))); }

// ---------------------------------------------------------------------------
// Forward.  Steps of 128 keys: S = Q K^T (tensor memory), p = 2^(c s - m) as bf16 beside it, O += p V.
// The row's reference m follows its running maximum only where that has grown by more than 8 (2^8 fits every type
// here): then O is multiplied in tensor memory, which otherwise stays with the MMAs.
// S is free again as soon as the rows have read it into registers: S of the next step, and of the next item, is formed under the
// exponentials of this one.  Half of an SM's tensor memory: two CTAs share an SM.  Each row has two threads (its warps are latency-bound:
// four warps to a scheduler instead of two), which agree on the reference when one of them needs a new one.
// ---------------------------------------------------------------------------
struct Fwd {
    static constexpr int kRowThreads = 2 * kRows, kThreads = kRowThreads + 64, kMma = 8, kLoad = 9, kWarps = 10, kPerSm = 2;
    static constexpr int Q = 0, K = 32768, V = K + 32768, bytes = V + 32768 + 1024;        // two places each; Q's take the finished tile
    static constexpr uint32_t kTmem = 256, cS = 0, cP = 128, cO = 192;
};

template <bool TAKES>
__global__ void __launch_bounds__(Fwd::kThreads, Fwd::kPerSm)
tc_win_fwd_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                  const __grid_constant__ CUtensorMap mapO, const __grid_constant__ WinArgs a, const __grid_constant__ ItemMap map, int* status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align1024(smem_raw);
    __shared__ __align__(16) Sched sched;
    __shared__ float s_top[2][kRows], s_sum[2][kRows];
    __shared__ unsigned s_bad[2][4];                      // a row's halves that are not finite, by warps
    __shared__ uint32_t s_redo[8];
    __shared__ uint64_t bar_q[2], free_q[2], bar_k[2], free_k[2], bar_v[2], free_v[2], bar_s, bar_read, bar_p, bar_o;
    __shared__ uint32_t tm_slot;
    const int tid = threadIdx.x, warp = warp_index();
    if (tid == 0) {
        cta_giveup_init();
        sched_init(sched, Fwd::kWarps);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar_q[i], 1); mbar_init(&free_q[i], 1); mbar_init(&bar_k[i], 1); mbar_init(&free_k[i], 1); mbar_init(&bar_v[i], 1); mbar_init(&free_v[i], 1);
        }
        mbar_init(&bar_s, 1); mbar_init(&bar_read, 8); mbar_init(&bar_p, 8); mbar_init(&bar_o, 1);
        mbar_fence_init();
    }
    if (tid < 8) s_redo[tid] = kNoItem;
    pdl_sync();
    if (!TAKES && blockIdx.x == 0 && tid == 0) *status = 0;
    if (warp == Fwd::kMma) { tmem_alloc(&tm_slot, Fwd::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tm_slot;
    auto tiles_of = [&](const Item& p) { return key_tiles(p.row0, (p.row0 + kRows < p.len ? p.row0 + kRows : p.len) - 1, a.window, a.sinks, 128); };
    // t: steps of all items so far
    if (warp == Fwd::kLoad) {
        bool ok = true;
        int t = 0, items = 0;
        for (int it = 0, index = blockIdx.x; index >= 0 && ok; ++it) {
            ok = __all_sync(0xffffffffu, sched_free(sched, it, status));
            if (!ok) break;
            if (elect_one()) sched_ask(sched, it, TAKES);
            const Item p = item_of(a, map, index);
            if (p.row0 < p.len) {
                const int buf = items & 1;
                if (items >= 2) ok = mbar_wait(&free_q[buf], (items / 2 - 1) & 1, status, kErrMma);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ++items;
                if (elect_one()) {
                    mbar_expect_tx(&bar_q[buf], 16384);
                    tma_load_4d(smem + Fwd::Q + buf * 16384, &mapQ, 0, p.row0, p.h, p.b, &bar_q[buf]);
                }
                const int hk = p.h / a.G;
                const bf16* V = (const bf16*)a.V + p.b * a.kb + hk * a.kh;
                const KeyTiles kt = tiles_of(p);
                for (int x = 0; x < kt.count(); ++x, ++t) {
                    const int k0 = kt.at(x) * 128, s = t & 1;
                    if (t >= 2) ok = mbar_wait(&free_k[s], (t / 2 - 1) & 1, status, kErrMma);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (elect_one()) {
                        mbar_expect_tx(&bar_k[s], 16384);
                        tma_load_4d(smem + Fwd::K + s * 16384, &mapK, 0, k0, hk, p.b, &bar_k[s]);
                    }
                    if (t >= 2) ok = mbar_wait(&free_v[s], (t / 2 - 1) & 1, status, kErrMma);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const bool ends = p.len < a.n && k0 + 128 > p.len;
                    if (ends) warp_load_tile<128>(smem + Fwd::V + s * 16384, V, a.kn, k0, p.len);
                    if (elect_one()) {
                        if (ends) {
                            mbar_arrive(&bar_v[s]);
                        } else {
                            mbar_expect_tx(&bar_v[s], 16384);
                            tma_load_4d(smem + Fwd::V + s * 16384, &mapV, 0, k0, hk, p.b, &bar_v[s]);
                        }
                    }
                }
                if (!ok) break;
            }
            index = sched_next(sched, it, TAKES, status);
            __syncwarp();
            if (tid % 32 == 0) sched_taken(sched, it);
        }
    } else if (warp == Fwd::kMma) {
        if (elect_one()) {
            constexpr uint32_t idesc_s = idesc_bf16(128, 128, false, false), idesc_o = idesc_bf16(128, 64, false, true);
            const uint64_t qd = smem_desc(smem_u32(smem + Fwd::Q), 0, 1024, kSwz128);
            const uint64_t kd = smem_desc(smem_u32(smem + Fwd::K), 0, 1024, kSwz128), vd = smem_desc(smem_u32(smem + Fwd::V), 0, 1024, kSwz128);
            bool ok = true, owed = false, first = false;              // the step before still has its product with V to come
            int t = 0, items = 0;
            auto product = [&](int y) {
                const int s = y & 1;
                ok = ok && mbar_wait(&bar_v[s], (y / 2) & 1, status, kErrTma) && mbar_wait(&bar_p, y & 1, status, kErrMma);
                owed = false;
                if (!ok) return;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < 8; ++k) umma_ts(tm + Fwd::cO, tm + Fwd::cP + k * 8, desc_off(vd, s * 16384 + k * 2048), idesc_o, (!first || k > 0) ? 1u : 0u);
                umma_commit(&bar_o);
                umma_commit(&free_v[s]);
            };
            for (int it = 0, index = blockIdx.x; index >= 0 && ok; ++it) {
                const Item p = item_of(a, map, index);
                if (p.row0 < p.len) {
                    const int steps = tiles_of(p).count(), buf = items & 1;
                    ok = mbar_wait(&bar_q[buf], (items / 2) & 1, status, kErrTma);
                    ++items;
                    for (int x = 0; x < steps && ok; ++x, ++t) {
                        const int s = t & 1;
                        ok = mbar_wait(&bar_k[s], (t / 2) & 1, status, kErrTma);
                        if (t > 0) ok = ok && mbar_wait(&bar_read, (t - 1) & 1, status, kErrMma);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_ss(tm + Fwd::cS, desc_off(qd, buf * 16384 + k * 32), desc_off(kd, s * 16384 + k * 32), idesc_s, k > 0);
                        umma_commit(&bar_s);
                        umma_commit(&free_k[s]);
                        if (owed) product(t - 1);
                        owed = true;
                        first = x == 0;
                    }
                } else if (owed) {
                    product(t - 1);                       // (nobody waits for an item that asks for nothing)
                }
                if (!ok) break;
                index = sched_next(sched, it, TAKES, status);
                sched_taken(sched, it);
            }
            if (ok && owed) product(t - 1);
        }
    } else {
        const int half = warp / 4, row = tid % kRows, lane = tid % 32, pair_bar = 1 + warp % 4;      // (the two warps of a row)
        const uint32_t lane_tm = tm + ((uint32_t)(warp % 4 * 32) << 16);
        const float c = a.c;
        const f2 c2 = pack2(c, c);
        bool ok = true, stored = false;                   // a finished tile may still be on its way out of the other place
        int t = 0, items = 0;
        for (int it = 0, index = blockIdx.x; index >= 0; ++it) {
            const Item p = item_of(a, map, index);
            const int i = p.row0 + row, i_first = p.row0 + warp % 4 * 32;
            float* lse = a.lse + ((int64_t)p.b * a.H + p.h) * a.n;
            if (p.row0 < p.len) {
                const KeyTiles kt = tiles_of(p);
                const int steps = kt.count();
                float m = neg_inf(), l = 0.f;
                for (int x = 0; x < steps; ++x, ++t) {
                    const int k0 = kt.at(x) * 128 + half * 64;
                    ok = mbar_wait(&bar_s, t & 1, status, kErrMma) && ok;
                    tc_fence_after();
                    Cols<32> s[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) s[q].load(lane_tm + Fwd::cS + half * 64 + q * 32);
                    tmem_ld_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar_read);
                    const bool whole = sees_all(i_first, k0, 64, a.window, a.sinks);
                    const KeyMask km = key_mask(i, k0, a.window, a.sinks);
                    Seen seen[2];
                    float tops[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t w = whole ? 0xffffffffu : km.word(q);
                        seen[q] = whole ? kAll : seen_by_warp(w);
                        tops[q] = neg_inf();
                        if (seen[q] == kNone) continue;
                        if (seen[q] == kSome) mask_scores(s[q], w);
                        float t1 = neg_inf();
#pragma unroll
                        for (int j = 0; j < 32; j += 4) { tops[q] = fmaxf(tops[q], fmaxf(s[q][j], s[q][j + 1])); t1 = fmaxf(t1, fmaxf(s[q][j + 2], s[q][j + 3])); }
                        tops[q] = fmaxf(tops[q], t1);
                    }
                    float top = fmaxf(tops[0], tops[1]), alpha = 1.f;
                    const bool any = bar_any(pair_bar, 64, (top - m) * c > 8.f);
                    if (any) {
                        s_top[half][row] = top;
                        bar_sync(pair_bar, 64);
                        top = fmaxf(top, s_top[1 - half][row]);
                        if ((top - m) * c > 8.f) { alpha = exp2_approx((m - top) * c); m = top; l *= alpha; }
                    }
                    if (x > 0) {                          // the weights of the step before have been used, O is complete up to it
                        ok = mbar_wait(&bar_o, (t - 1) & 1, status, kErrMma) && ok;
                        tc_fence_after();
                        if (any) {
#pragma unroll 1
                            for (int q = 0; q < 2; ++q) {
                                uint32_t o[16];
                                tmem_ld16(lane_tm + Fwd::cO + half * 32 + q * 16, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                                tmem_st16(lane_tm + Fwd::cO + half * 32 + q * 16, o);
                            }
                        }
                    }
                    const float base = m == neg_inf() ? 0.f : m * c;
                    const f2 base2 = pack2(-base, -base);
                    f2 sum = 0;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t to = lane_tm + Fwd::cP + half * 32 + q * 16;
                        if (seen[q] == kNone) { store_zeros(to); continue; }
                        uint32_t pk[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const f2 e = exp2_pair(fma2(s[q].pair(j), c2, base2));
                            sum = add2(sum, e);
                            pk[j / 2] = pack_bf16(lo2(e), hi2(e));
                        }
                        tmem_st16(to, pk);
                    }
                    l += lo2(sum) + hi2(sum);
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar_p);
                    if (tid == 0 && stored) { bulk_wait_read(); mbar_arrive(&free_q[(items - 1) & 1]); }
                    stored = false;
                }
                uint8_t* st = smem + Fwd::Q + (items & 1) * 16384;
                ++items;
                s_sum[half][row] = l;
                bar_sync(pair_bar, 64);
                l += s_sum[1 - half][row];                // (two summands: the same in both threads)
                const bool live = i < p.len;
                const float v = (m * c + log2f(l)) * kLn2;
                ok = mbar_wait(&bar_o, (t - 1) & 1, status, kErrMma) && ok;
                tc_fence_after();
                const bool fine = stage_half(st, row, half, lane_tm + Fwd::cO, 1.f / l, live) || !finite(v);      // (where v is not, the row is NaN)
                tc_fence_before();
                if (ok && half == 0 && i < a.n) lse[i] = live ? v : neg_inf();
                const unsigned bad = __ballot_sync(0xffffffffu, ok && !fine && live);
                if (lane == 0) s_bad[half][warp % 4] = bad;
                fence_proxy_async_smem();
                bar_sync(5, Fwd::kRowThreads);
                // (each of a row's two warps takes every other one)
                redo_note(a.redo + (size_t)index * 8 + warp, index, (s_bad[0][warp % 4] | s_bad[1][warp % 4]) & (half ? 0xaaaaaaaau : 0x55555555u), s_redo[warp]);
                if (tid == 0 && !cta_gave_up()) { tma_store_4d(&mapO, st, 0, p.row0, p.h, p.b); bulk_commit(); }
                stored = true;
            } else {                                      // behind the sequence's end
                zero_tile<Fwd::kRowThreads>((bf16*)a.out + p.b * a.qb + p.h * a.qh, a.qn, p.row0, a.n, tid);
                if (half == 0 && i < a.n) lse[i] = neg_inf();
            }
            index = sched_next(sched, it, TAKES, status);
            if (bar_any(5, Fwd::kRowThreads, index < 0)) index = -1;        // (all of them or none: they share barriers)
            if (lane == 0) sched_taken(sched, it);
        }
        if (tid == 0) bulk_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == Fwd::kMma) { cta_teardown_warp(); tmem_dealloc(tm, Fwd::kTmem); }
    if (warp < 8 && !cta_gave_up())
        redo_noted(s_redo[warp], [&](uint32_t code) { return a.redo + (size_t)code * 8 + warp; }, [&](uint32_t code, int k) {
            const Item p = item_of(a, map, code);
            const int r = p.row0 + warp % 4 * 32 + k, hk = p.h / a.G;
            const bf16 *K = (const bf16*)a.K + p.b * a.kb + hk * a.kh, *V = (const bf16*)a.V + p.b * a.kb + hk * a.kh;
            const int64_t at = p.b * a.qb + p.h * a.qh + r * a.qn;
            if (row_tainted(K, V, a.kn, r, a.window, a.sinks, p.len))
                st2((bf16*)a.out + at + 2 * (tid % 32), redo_out_row((const bf16*)a.Q + at, K, V, a.kn, r, a.window, a.sinks, a.c));
        });
}

// ---------------------------------------------------------------------------
// Backward: one CTA per SM, three warpgroups that take its steps in turn, each with a buffer of scores and dP that its
// p and ds take the place of.  (MMAs complete in the order of their issue: the scores of step t + 3 follow the products of step t.)
// The sums of an item stay in tensor memory until the warpgroups that finish it have read them; the others go on with the next one.
// ---------------------------------------------------------------------------
constexpr int kGroups = 3;

// The MMA lane's account of steps: products follow the scores by up to three steps, and by no item more than the present one (an item that
// waits for its last products must not wait for the next answer of the scheduler).
struct Steps {
    int t = 0, done = 0;              // steps with scores, with products
    int started = 0;                  // items with products
    uint32_t first = 0, last = 0;     // of the steps between: the first, the last of their item (bit: step mod 3)
    __device__ __forceinline__ void add(bool is_first, bool is_last) {
        const uint32_t b = 1u << (t % kGroups);
        first = is_first ? first | b : first & ~b;
        last = is_last ? last | b : last & ~b;
        ++t;
    }
    __device__ __forceinline__ bool owes_first() const { return (first >> (done % kGroups)) & 1u; }
    __device__ __forceinline__ bool owes_last() const { return (last >> (done % kGroups)) & 1u; }
};

// ---------------------------------------------------------------------------
// Query side.  Steps of 64 keys: S = Q K^T and dP = dO V^T into tensor memory, ds = p (dP - D) as bf16 over S, dQ += ds K.
// Every thread forms D0_i = do_i . o_i of its row from the tiles in shared memory, with o as it was stored, rounded to bf16.  What that takes from D
// shows in the sum of the row's ds, which is D - D0 (the weights sum to one), and with D0 alone it is as large as all other roundings
// together where few keys count (windows of 8 rows: 2.6e-3 instead of 2.3e-3; of 2: 3.6e-3).  So p goes over dP as a second operand, Kb += p K,
// and dQ = sum ds k - (D - D0) Kb; the key side gets -lse log2(e) and the whole -D.  Sixteen MMAs a step instead of twelve:
// 192 heads x 8192 rows, window 512, 586 us instead of 538.
// ---------------------------------------------------------------------------
struct Dq {
    static constexpr int kMma = 12, kLoad = 13, kWarps = 14, kThreads = 32 * kWarps, kStages = 5;
    static constexpr int QGO = 0, KV = 2 * 49152, St = KV + kStages * 16384, bytes = St + kGroups * 16384 + 1024;
    static constexpr uint32_t kTmem = 512, cDq = 0, cS = 64, cKb = 448;        // cS + 128 warpgroup: S (ds), dP (p)
};

template <bool TAKES>
__global__ void __launch_bounds__(Dq::kThreads, 1)
tc_win_dq_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapG, const __grid_constant__ CUtensorMap mapO,
                 const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ CUtensorMap mapDq, const __grid_constant__ WinArgs a,
                 const __grid_constant__ ItemMap map, int* status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align1024(smem_raw);
    __shared__ __align__(16) Sched sched;
    __shared__ float s_lse[2][kRows];
    __shared__ uint32_t s_redo[4 * kGroups];
    __shared__ uint64_t bar_q[2], free_q[2], bar_kv[Dq::kStages], free_kv[Dq::kStages], bar_s[kGroups], bar_ds[kGroups], bar_fin[4], bar_sum[4], bar_acc;
    __shared__ uint32_t tm_slot;
    const int tid = threadIdx.x, warp = warp_index(), lane = tid % 32;
    if (tid == 0) {
        cta_giveup_init();
        sched_init(sched, Dq::kWarps);
        for (int i = 0; i < 4; ++i) mbar_init(&bar_sum[i], 4 * kGroups);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_q[i], 33); mbar_init(&free_q[i], 1 + 4 * kGroups); }
        for (int i = 0; i < Dq::kStages; ++i) { mbar_init(&bar_kv[i], 1); mbar_init(&free_kv[i], 1); }
        for (int i = 0; i < kGroups; ++i) { mbar_init(&bar_s[i], 1); mbar_init(&bar_ds[i], 4); }
        for (int i = 0; i < 4; ++i) mbar_init(&bar_fin[i], 1);
        mbar_init(&bar_acc, 4);
        mbar_fence_init();
    }
    if (tid < 4 * kGroups) s_redo[tid] = kNoItem;
    pdl_sync();
    if (!TAKES && blockIdx.x == 0 && tid == 0) *status = 0;
    if (warp == Dq::kMma) { tmem_alloc(&tm_slot, Dq::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tm_slot;
    auto tiles_of = [&](const Item& p) { return key_tiles(p.row0, (p.row0 + kRows < p.len ? p.row0 + kRows : p.len) - 1, a.window, a.sinks, 64); };
    if (warp == Dq::kLoad) {
        bool ok = true;
        int t = 0, items = 0;                             // items: with Q, dO, O asked for, one ahead of the keys (8192 rows of 192 heads 3 % faster)
        auto load_q = [&](const Item& p) {
            const int buf = items & 1;
            if (items >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&free_q[buf], (items / 2 - 1) & 1, status, kErrMma));
            if (!ok) return;
            ++items;
            if (elect_one()) {
                mbar_expect_tx(&bar_q[buf], 49152);
                tma_load_4d(smem + Dq::QGO + buf * 49152, &mapQ, 0, p.row0, p.h, p.b, &bar_q[buf]);
                tma_load_4d(smem + Dq::QGO + buf * 49152 + 16384, &mapG, 0, p.row0, p.h, p.b, &bar_q[buf]);
                tma_load_4d(smem + Dq::QGO + buf * 49152 + 32768, &mapO, 0, p.row0, p.h, p.b, &bar_q[buf]);
            }
            const int64_t soff = ((int64_t)p.b * a.H + p.h) * a.n + p.row0;
#pragma unroll
            for (int e = lane; e < kRows; e += 32) {
                const int bytes = p.row0 + e < p.len ? 4 : 0;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(&s_lse[buf][e])), "l"(a.lse_in + (bytes ? soff + e : 0)), "r"(bytes) : "memory");
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&bar_q[buf])) : "memory");
        };
        int index = blockIdx.x;
        Item p = item_of(a, map, index);
        if (p.row0 < p.len) load_q(p);
        for (int it = 0; index >= 0 && ok; ++it) {
            ok = __all_sync(0xffffffffu, sched_free(sched, it, status));
            if (!ok) break;
            if (elect_one()) sched_ask(sched, it, TAKES);
            Item ahead = p;
            auto look_ahead = [&]() {
                index = sched_next(sched, it, TAKES, status);
                __syncwarp();
                if (lane == 0) sched_taken(sched, it);
                if (index < 0) return;
                ahead = item_of(a, map, index);
                if (ahead.row0 < ahead.len) load_q(ahead);
            };
            if (p.row0 < p.len) {
                const int hk = p.h / a.G;
                const int64_t koff = p.b * a.kb + hk * a.kh;
                const KeyTiles kt = tiles_of(p);
                const int steps = kt.count();
                for (int x = 0; x < steps; ++x, ++t) {
                    const int k0 = kt.at(x) * 64, s = t % Dq::kStages;
                    if (t >= Dq::kStages) ok = mbar_wait(&free_kv[s], (t / Dq::kStages - 1) & 1, status, kErrMma);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    uint8_t* st = smem + Dq::KV + s * 16384;
                    const bool ends = p.len < a.n && k0 + 64 > p.len;
                    if (ends) {
                        warp_load_tile<64>(st, (const bf16*)a.K + koff, a.kn, k0, p.len);
                        warp_load_tile<64>(st + 8192, (const bf16*)a.V + koff, a.kn, k0, p.len);
                    }
                    if (elect_one()) {
                        if (ends) {
                            mbar_arrive(&bar_kv[s]);
                        } else {
                            mbar_expect_tx(&bar_kv[s], 16384);
                            tma_load_4d(st, &mapK, 0, k0, hk, p.b, &bar_kv[s]);
                            tma_load_4d(st + 8192, &mapV, 0, k0, hk, p.b, &bar_kv[s]);
                        }
                    }
                    if (x == (steps > 2 ? 2 : steps - 1)) look_ahead();
                    if (!ok) break;
                }
            } else {
                look_ahead();
            }
            p = ahead;
        }
    } else if (warp == Dq::kMma) {
        if (elect_one()) {
            constexpr uint32_t idesc_s = idesc_bf16(128, 64, false, false), idesc_o = idesc_bf16(128, 64, false, true);
            const uint64_t qgd = smem_desc(smem_u32(smem + Dq::QGO), 0, 1024, kSwz128), kvd = smem_desc(smem_u32(smem + Dq::KV), 0, 1024, kSwz128);
            bool ok = true;
            int items = 0;
            Steps w;
            auto product = [&]() {
                const int g = w.done % kGroups, s = w.done % Dq::kStages;
                const bool first = w.owes_first(), last = w.owes_last();
                ok = ok && mbar_wait(&bar_ds[g], (w.done / kGroups) & 1, status, kErrMma);
                // the sum of the item before has been read
                if (first && w.started++ > 0) ok = ok && mbar_wait(&bar_acc, (w.started - 2) & 1, status, kErrMma);
                ++w.done;
                if (!ok) return;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_ts(tm + Dq::cDq, tm + Dq::cS + g * 128 + k * 8, desc_off(kvd, s * 16384 + k * 2048), idesc_o, (!first || k > 0) ? 1u : 0u);
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_ts(tm + Dq::cKb, tm + Dq::cS + g * 128 + 64 + k * 8, desc_off(kvd, s * 16384 + k * 2048), idesc_o, (!first || k > 0) ? 1u : 0u);
                umma_commit(&free_kv[s]);
                if (last) umma_commit(&bar_fin[(w.started - 1) & 3]);
            };
            for (int it = 0, index = blockIdx.x; index >= 0 && ok; ++it) {
                const Item p = item_of(a, map, index);
                const int begun = w.t;
                if (p.row0 < p.len) {
                    const int steps = tiles_of(p).count(), buf = items & 1;
                    ok = mbar_wait(&bar_q[buf], (items / 2) & 1, status, kErrTma);
                    ++items;
                    for (int x = 0; x < steps && ok; ++x) {
                        if (w.t - w.done == kGroups) product();
                        const int g = w.t % kGroups, s = w.t % Dq::kStages;
                        ok = ok && mbar_wait(&bar_kv[s], (w.t / Dq::kStages) & 1, status, kErrTma);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_ss(tm + Dq::cS + g * 128, desc_off(qgd, buf * 49152 + k * 32), desc_off(kvd, s * 16384 + k * 32), idesc_s, k > 0);
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_ss(tm + Dq::cS + g * 128 + 64, desc_off(qgd, buf * 49152 + 16384 + k * 32), desc_off(kvd, s * 16384 + 8192 + k * 32), idesc_s, k > 0);
                        umma_commit(&bar_s[g]);
                        if (x + 1 == steps) umma_commit(&free_q[buf]);
                        w.add(x == 0, x + 1 == steps);
                    }
                }
                while (ok && w.done < begun) product();
                if (!ok) break;
                index = sched_next(sched, it, TAKES, status);
                sched_taken(sched, it);
            }
            while (ok && w.done < w.t) product();
        }
    } else {
        const int group = warp / 4, row = tid % kRows;
        const uint32_t lane_tm = tm + ((uint32_t)(warp % 4 * 32) << 16), tS = lane_tm + Dq::cS + group * 128;
        const f2 c2 = pack2(a.c, a.c);
        uint8_t* st = smem + Dq::St + group * 16384;
        bool ok = true;
        int t = group, t0 = 0, items = 0;                 // this warpgroup's next step, the item's first
        for (int it = 0, index = blockIdx.x; index >= 0; ++it) {
            const Item p = item_of(a, map, index);
            const int i = p.row0 + row, i_first = p.row0 + warp % 4 * 32;
            const int64_t qoff = p.b * a.qb + p.h * a.qh;
            if (p.row0 < p.len) {
                const KeyTiles kt = tiles_of(p);
                const int end = t0 + kt.count();
                const int buf = items & 1;
                ok = mbar_wait(&bar_q[buf], (items / 2) & 1, status, kErrTma) && ok;
                float2 stat = make_float2(-s_lse[buf][row] * kLog2e, 0.f);         // -lse log2(e), -D
                const uint8_t *gt = smem + Dq::QGO + buf * 49152 + 16384, *ot = gt + 16384;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint4 o = *reinterpret_cast<const uint4*>(ot + swz128_offset(row, k)), g = *reinterpret_cast<const uint4*>(gt + swz128_offset(row, k));
                    const uint32_t ow[4] = {o.x, o.y, o.z, o.w}, gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        stat.y = fmaf(__uint_as_float(gw[w] << 16), -__uint_as_float(ow[w] << 16), stat.y);
                        stat.y = fmaf(__uint_as_float(gw[w] & 0xffff0000u), -__uint_as_float(ow[w] & 0xffff0000u), stat.y);
                    }
                }
                const int64_t at = ((int64_t)p.b * a.H + p.h) * a.n + i, rows = (int64_t)a.B * a.H * a.n;
                f2 sum = 0;
                const f2 l2 = pack2(stat.x, stat.x), D2 = pack2(stat.y, stat.y);
                __syncwarp();
                if (lane == 0) mbar_arrive(&free_q[buf]);
                for (; t < end; t += kGroups) {
                    const int k0 = kt.at(t - t0) * 64;
                    ok = mbar_wait(&bar_s[group], (t / kGroups) & 1, status, kErrMma) && ok;
                    tc_fence_after();
                    const bool whole = sees_all(i_first, k0, 64, a.window, a.sinks);
                    const KeyMask km = key_mask(i, k0, a.window, a.sinks);
#pragma unroll 1
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t w = whole ? 0xffffffffu : km.word(q);
                        const Seen seen = whole ? kAll : seen_by_warp(w);
                        if (seen == kNone) { store_zeros(tS + q * 16); store_zeros(tS + 64 + q * 16); continue; }
                        Cols<32> s, d;
                        s.load(tS + q * 32);
                        d.load(tS + 64 + q * 32);
                        tmem_ld_wait();
                        // (a weight of 0 times an infinity in dP is NaN, and the row is formed again)
                        if (seen == kSome) mask_scores(s, w);
                        uint32_t pk[16], dk[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const f2 pr = exp2_pair(fma2(s.pair(j), c2, l2)), ds = mul2(pr, add2(d.pair(j), D2));
                            sum = add2(sum, ds);
                            pk[j / 2] = pack_bf16(lo2(pr), hi2(pr));
                            dk[j / 2] = pack_bf16(lo2(ds), hi2(ds));
                        }
                        tmem_st16(tS + q * 16, dk);
                        tmem_st16(tS + 64 + q * 16, pk);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar_ds[group]);
                }
                // The warpgroup with the last step finishes the item; the others leave it their sums of ds (which steps those are of depends on the
                // distance from the last step alone, and so does their order).  A warpgroup may be two items ahead of another, not three (it would need
                // an answer of the scheduler that the other has not taken yet): hence four barriers, as for the products.
                const int behind = (group - (end - 1) % kGroups + kGroups) % kGroups;        // 0: it finishes, 2: the step before the last
                float r = lo2(sum) + hi2(sum);
                if (behind > 0 && i < p.len) a.stat_r[(behind - 1) * rows + at] = r;
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_sum[items & 3]);
                if (behind == 0) {
                    if (row == 0) bulk_wait_read();
                    ok = mbar_wait(&bar_sum[items & 3], (items / 4) & 1, status, kErrMma) && ok;
                    if (ok && i < p.len) {
                        r += a.stat_r[rows + at] + a.stat_r[at];
                        r = finite(r) ? r : 0.f;          // (an infinity in a pair that does not count is in it too)
                        a.stat_l[at] = stat.x;
                        a.stat_d[at] = stat.y -= r;
                    }
                    ok = mbar_wait(&bar_fin[items & 3], (items / 4) & 1, status, kErrMma) && ok;
                    tc_fence_after();
                    bar_sync(1 + group, kRows);
                    const bool live = i < p.len, fine = stage_row(st, row, lane_tm + Dq::cDq, a.scale, live, lane_tm + Dq::cKb, -r * a.scale);
                    tc_fence_before();
                    const unsigned bad = __ballot_sync(0xffffffffu, ok && !fine && live && stat.x == stat.x && stat.y == stat.y);      // (with a NaN there the row is NaN)
                    if (lane == 0) mbar_arrive(&bar_acc);
                    redo_note(a.redo + (size_t)index * 4 + warp % 4, index, bad, s_redo[warp]);
                    fence_proxy_async_smem();
                    bar_sync(1 + group, kRows);
                    if (row == 0 && !cta_gave_up()) { tma_store_4d(&mapDq, st, 0, p.row0, p.h, p.b); bulk_commit(); }
                }
                t0 = end;
                ++items;
            } else if (group == 0) {
                zero_tile<kRows>((bf16*)a.dQ + qoff, a.qn, p.row0, a.n, row);
            }
            index = sched_next(sched, it, TAKES, status);
            if (bar_any(1 + group, kRows, index < 0)) index = -1;            // (a whole warpgroup or none of it: it shares barriers)
            if (lane == 0) sched_taken(sched, it);
        }
        if (row == 0) bulk_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == Dq::kMma) { cta_teardown_warp(); tmem_dealloc(tm, Dq::kTmem); }
    if (warp < 4 * kGroups && !cta_gave_up())
        redo_noted(s_redo[warp], [&](uint32_t code) { return a.redo + (size_t)code * 4 + warp % 4; }, [&](uint32_t code, int k) {
            const Item p = item_of(a, map, code);
            const int r = p.row0 + warp % 4 * 32 + k, hk = p.h / a.G;
            const bf16 *K = (const bf16*)a.K + p.b * a.kb + hk * a.kh, *V = (const bf16*)a.V + p.b * a.kb + hk * a.kh;
            const int64_t at = p.b * a.qb + p.h * a.qh + r * a.qn, stat = ((int64_t)p.b * a.H + p.h) * a.n + r;
            if (row_tainted(K, V, a.kn, r, a.window, a.sinks, p.len))
                st2((bf16*)a.dQ + at + 2 * lane, redo_dq_row((const bf16*)a.Q + at, (const bf16*)a.dO + at, K, V, a.kn, r, a.window, a.sinks, a.c, a.scale,
                                                            make_float2(-a.stat_l[stat], -a.stat_d[stat])));
        });
}

// ---------------------------------------------------------------------------
// Key side: one tile of 128 keys (thread = key), steps of 64 query rows of every query head that shares the key head:
// S^T = K Q^T, dP^T = V dO^T, p^T and ds^T as bf16 over them, dV += p^T dO, dK += ds^T Q.
// ---------------------------------------------------------------------------
struct Dkv {
    static constexpr int kMma = 12, kLoad = 13, kWarps = 14, kThreads = 32 * kWarps, kStages = 6;
    static constexpr int KV = 0, QG = 65536, St = QG + kStages * 16384, bytes = St + kGroups * 16384 + 1024;
    static constexpr uint32_t kTmem = 512, cDk = 0, cDv = 64, cS = 128;        // cS + 128 warpgroup: S (p), dP (ds)
};

// PARTS: there are items that are parts of the sinks' tiles, or key heads in several (the code for them costs others 4 %: 699 against 674 us on 8192 rows of 16 x 12 heads)
template <bool PARTS>
__global__ void __launch_bounds__(Dkv::kThreads, 1)
tc_win_dkv_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const __grid_constant__ CUtensorMap mapQ,
                  const __grid_constant__ CUtensorMap mapG, const __grid_constant__ CUtensorMap mapDk, const __grid_constant__ CUtensorMap mapDv,
                  const __grid_constant__ WinArgs a, const __grid_constant__ ItemMap map, int* status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = align1024(smem_raw);
    __shared__ __align__(16) Sched sched;
    __shared__ __align__(16) float s_stat[Dkv::kStages][2][64];          // -lse log2(e), -D
    __shared__ uint32_t s_redo[4 * kGroups];
    __shared__ uint64_t bar_kv[2], free_kv[2], bar_qg[Dkv::kStages], free_qg[Dkv::kStages], bar_s[kGroups], bar_ds[kGroups], bar_fin[4], bar_acc;
    __shared__ uint32_t tm_slot;
    const int tid = threadIdx.x, warp = warp_index(), lane = tid % 32;
    if (tid == 0) {
        cta_giveup_init();
        sched_init(sched, Dkv::kWarps);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_kv[i], 1); mbar_init(&free_kv[i], 1); }
        for (int i = 0; i < Dkv::kStages; ++i) { mbar_init(&bar_qg[i], 33); mbar_init(&free_qg[i], 1); }
        for (int i = 0; i < kGroups; ++i) { mbar_init(&bar_s[i], 1); mbar_init(&bar_ds[i], 4); }
        for (int i = 0; i < 4; ++i) mbar_init(&bar_fin[i], 1);
        mbar_init(&bar_acc, 8);
        mbar_fence_init();
    }
    if (tid < 4 * kGroups) s_redo[tid] = kNoItem;
    pdl_sync();
    if (warp == Dkv::kMma) { tmem_alloc(&tm_slot, Dkv::kTmem); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tm_slot;
    auto item = [&](int index) {
        if constexpr (PARTS) {
            return key_item(a, index, kRows, [&](int x) { return (int)map.tiles.div(x); }, [&](int x) { return (int)map.heads.div(x); },
                            [&](int x) { return (int)map.parts.div(x); });
        } else {
            const Item q = item_of(a, map, index);
            return KeyItem{q.b, q.h, q.row0, q.len, q.row0, q.len, -1};
        }
    };
    auto tiles_of = [&](const KeyItem& p) { return (p.end(a, kRows) - p.begin + 63) / 64; };       // steps per query head
    // where a row's gradients (0: dK, 1: dV) are added up from
    auto sum_place = [&](const KeyItem& p, int which, int r) -> float* {
        if (p.part >= 0 && r < a.sinks) return partial_row(a, p.b, p.h, p.part, which, r);
        return p.part <= 0 && a.hs > 1 ? sum_row(a, p.b, p.h, which, p.key0 + r) : nullptr;
    };
    if (warp == Dkv::kLoad) {
        bool ok = true;
        int t = 0, items = 0;
        for (int it = 0, index = blockIdx.x; index >= 0 && ok; ++it) {
            ok = __all_sync(0xffffffffu, sched_free(sched, it, status));
            if (!ok) break;
            if (elect_one()) sched_ask(sched, it, true);
            const KeyItem p = item(index);
            if (!p.empty()) {
                const int kv = items & 1, tiles = tiles_of(p), steps = tiles * a.G;
                if (items >= 2) ok = mbar_wait(&free_kv[kv], (items / 2 - 1) & 1, status, kErrMma);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ++items;
                if (elect_one()) {
                    mbar_expect_tx(&bar_kv[kv], 32768);
                    const int hk = PARTS ? p.h / a.hs : p.h;
                    tma_load_4d(smem + Dkv::KV + kv * 32768, &mapK, 0, p.key0, hk, p.b, &bar_kv[kv]);
                    tma_load_4d(smem + Dkv::KV + kv * 32768 + 16384, &mapV, 0, p.key0, hk, p.b, &bar_kv[kv]);
                }
                for (int x = 0, h = p.h * a.G, i0 = p.begin; x < steps; ++x, ++t, i0 += 64) {
                    const int s = t % Dkv::kStages;
                    if (i0 - p.begin == tiles * 64) { i0 = p.begin; ++h; }
                    if (t >= Dkv::kStages) ok = mbar_wait(&free_qg[s], (t / Dkv::kStages - 1) & 1, status, kErrMma);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    uint8_t* st = smem + Dkv::QG + s * 16384;
                    const bool ends = p.len < a.n && i0 + 64 > p.len;
                    if (ends) {
                        const int64_t off = p.b * a.qb + h * a.qh;
                        warp_load_tile<64>(st, (const bf16*)a.Q + off, a.qn, i0, p.len);
                        warp_load_tile<64>(st + 8192, (const bf16*)a.dO + off, a.qn, i0, p.len);
                    }
                    if (elect_one()) {
                        if (ends) {
                            mbar_arrive(&bar_qg[s]);
                        } else {
                            mbar_expect_tx(&bar_qg[s], 16384);
                            tma_load_4d(st, &mapQ, 0, i0, h, p.b, &bar_qg[s]);
                            tma_load_4d(st + 8192, &mapG, 0, i0, h, p.b, &bar_qg[s]);
                        }
                    }
                    // the rows' statistics (zeros behind the end), two rows a lane
                    const int64_t soff = ((int64_t)p.b * a.H + h) * a.n + i0;
#pragma unroll
                    for (int e = lane; e < 64; e += 32) {
                        const int bytes = i0 + e < p.len ? 4 : 0;
                        const int64_t at = bytes ? soff + e : 0;
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(&s_stat[s][0][e])), "l"(a.stat_l + at), "r"(bytes) : "memory");
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(&s_stat[s][1][e])), "l"(a.stat_d + at), "r"(bytes) : "memory");
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&bar_qg[s])) : "memory");
                }
                if (!ok) break;
            }
            index = sched_next(sched, it, true, status);
            __syncwarp();
            if (lane == 0) sched_taken(sched, it);
        }
    } else if (warp == Dkv::kMma) {
        if (elect_one()) {
            constexpr uint32_t idesc_s = idesc_bf16(128, 64, false, false), idesc_o = idesc_bf16(128, 64, false, true);
            const uint64_t kvd = smem_desc(smem_u32(smem + Dkv::KV), 0, 1024, kSwz128), qgd = smem_desc(smem_u32(smem + Dkv::QG), 0, 1024, kSwz128);
            bool ok = true;
            int items = 0;
            Steps w;
            auto product = [&]() {
                const int g = w.done % kGroups, s = w.done % Dkv::kStages;
                const bool first = w.owes_first(), last = w.owes_last();
                ok = ok && mbar_wait(&bar_ds[g], (w.done / kGroups) & 1, status, kErrMma);
                if (first && w.started++ > 0) ok = ok && mbar_wait(&bar_acc, (w.started - 2) & 1, status, kErrMma);
                ++w.done;
                if (!ok) return;
                tc_fence_after();
                const uint32_t ps = tm + Dkv::cS + g * 128;
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_ts(tm + Dkv::cDv, ps + k * 8, desc_off(qgd, s * 16384 + 8192 + k * 2048), idesc_o, (!first || k > 0) ? 1u : 0u);
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_ts(tm + Dkv::cDk, ps + 64 + k * 8, desc_off(qgd, s * 16384 + k * 2048), idesc_o, (!first || k > 0) ? 1u : 0u);
                umma_commit(&free_qg[s]);
                if (last) umma_commit(&bar_fin[(w.started - 1) & 3]);
            };
            for (int it = 0, index = blockIdx.x; index >= 0 && ok; ++it) {
                const KeyItem p = item(index);
                const int begun = w.t;
                if (!p.empty()) {
                    const int kv = items & 1, steps = tiles_of(p) * a.G;
                    ok = mbar_wait(&bar_kv[kv], (items / 2) & 1, status, kErrTma);
                    ++items;
                    for (int x = 0; x < steps && ok; ++x) {
                        if (w.t - w.done == kGroups) product();
                        const int g = w.t % kGroups, s = w.t % Dkv::kStages;
                        ok = ok && mbar_wait(&bar_qg[s], (w.t / Dkv::kStages) & 1, status, kErrTma);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_ss(tm + Dkv::cS + g * 128, desc_off(kvd, kv * 32768 + k * 32), desc_off(qgd, s * 16384 + k * 32), idesc_s, k > 0);
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_ss(tm + Dkv::cS + g * 128 + 64, desc_off(kvd, kv * 32768 + 16384 + k * 32), desc_off(qgd, s * 16384 + 8192 + k * 32), idesc_s, k > 0);
                        umma_commit(&bar_s[g]);
                        if (x + 1 == steps) umma_commit(&free_kv[kv]);
                        w.add(x == 0, x + 1 == steps);
                    }
                }
                while (ok && w.done < begun) product();
                if (!ok) break;
                index = sched_next(sched, it, true, status);
                sched_taken(sched, it);
            }
            while (ok && w.done < w.t) product();
        }
    } else {
        const int group = warp / 4, row = tid % kRows;
        const uint32_t lane_tm = tm + ((uint32_t)(warp % 4 * 32) << 16), tS = lane_tm + Dkv::cS + group * 128;
        const f2 c2 = pack2(a.c, a.c);
        uint8_t* st = smem + Dkv::St + group * 16384;
        bool ok = true;
        int t = group, t0 = 0, items = 0;
        for (int it = 0, index = blockIdx.x; index >= 0; ++it) {
            const KeyItem p = item(index);
            const int j = p.key0 + row, j_first = p.key0 + warp % 4 * 32;
            if (!p.empty()) {
                const int rows = tiles_of(p) * 64, end = t0 + rows / 64 * a.G;
                const int64_t past = (int64_t)j + a.window;
                const int last_row = ((j < a.sinks || past > p.len) ? p.len : (int)past) - 1;      // the last query row that sees this key
                int off = (t - t0) * 64;                  // of the step's first row from the item's
                for (; t < end; t += kGroups, off += kGroups * 64) {
                    while (off >= rows) off -= rows;      // (the next head's rows)
                    const int i0 = p.begin + off, stage = t % Dkv::kStages;
                    ok = mbar_wait(&bar_qg[stage], (t / Dkv::kStages) & 1, status, kErrTma) && ok;     // (the rows' statistics)
                    ok = mbar_wait(&bar_s[group], (t / kGroups) & 1, status, kErrMma) && ok;
                    tc_fence_after();
                    // (the same for the warp:) all of these rows see all of its keys
                    const bool whole = j_first + 31 <= i0 && i0 + 63 < p.len && (i0 + 63 - j_first < a.window || j_first + 31 < a.sinks);
                    const int lo = j - i0, hi = last_row - i0;
#pragma unroll 1
                    for (int q = 0; q < 2; ++q) {
                        const uint32_t w = whole ? 0xffffffffu : bits_below(hi + 1 - 32 * q) & ~bits_below(lo - 32 * q);
                        const Seen seen = whole ? kAll : seen_by_warp(w);
                        if (seen == kNone) { store_zeros(tS + q * 16); store_zeros(tS + 64 + q * 16); continue; }
                        Cols<32> s, d;
                        s.load(tS + q * 32);
                        d.load(tS + 64 + q * 32);
                        tmem_ld_wait();
                        if (seen == kSome) mask_scores(s, w);
                        const float *sl = &s_stat[stage][0][q * 32], *sd = &s_stat[stage][1][q * 32];
                        uint32_t pk[16], dk[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const ulonglong2 L = *reinterpret_cast<const ulonglong2*>(sl + e), D = *reinterpret_cast<const ulonglong2*>(sd + e);
#pragma unroll
                            for (int k = 0; k < 4; k += 2) {
                                const f2 pr = exp2_pair(fma2(s.pair(e + k), c2, k == 0 ? L.x : L.y)), ds = mul2(pr, add2(d.pair(e + k), k == 0 ? D.x : D.y));
                                pk[(e + k) / 2] = pack_bf16(lo2(pr), hi2(pr));
                                dk[(e + k) / 2] = pack_bf16(lo2(ds), hi2(ds));
                            }
                        }
                        tmem_st16(tS + q * 16, pk);
                        tmem_st16(tS + 64 + q * 16, dk);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar_ds[group]);
                }
                // The warpgroup with the last step finishes dK, the one before it dV: the third has the next item's first step, whose
                // products wait for these two (with that one finishing dV 674 us on 8192 rows of 192 heads).
                const bool has_k = (end - 1) % kGroups == group;
                if (has_k || (end + 1) % kGroups == group) {
                    if (row == 0) bulk_wait_read();
                    ok = mbar_wait(&bar_fin[items & 3], (items / 4) & 1, status, kErrMma) && ok;
                    tc_fence_after();
                    bar_sync(1 + group, kRows);
                    const bool live = j < p.len;
                    const uint32_t from = lane_tm + (has_k ? Dkv::cDk : Dkv::cDv);
                    const float f = has_k ? a.scale : 1.f;
                    if (PARTS) {
                        float* to = live && ok ? sum_place(p, has_k ? 0 : 1, row) : nullptr;
                        if (__any_sync(0xffffffffu, to != nullptr)) store_partial(to, from, f, to != nullptr);
                    }
                    if (PARTS && p.part > 0) {
                        tc_fence_before();
                        if (lane == 0) mbar_arrive(&bar_acc);
                    } else {
                        const bool fine = stage_row(st, row, from, f, live);
                        tc_fence_before();
                        const unsigned bad = __ballot_sync(0xffffffffu, ok && !fine && live);
                        if (lane == 0) mbar_arrive(&bar_acc);
                        const uint32_t code = 2 * (uint32_t)index + (has_k ? 0 : 1);
                        redo_note(a.redo + (size_t)code * 4 + warp % 4, code, bad, s_redo[warp]);
                        fence_proxy_async_smem();
                        bar_sync(1 + group, kRows);
                        if (row == 0 && !cta_gave_up() && (!PARTS || a.hs == 1)) { tma_store_4d(has_k ? &mapDk : &mapDv, st, 0, p.key0, p.h, p.b); bulk_commit(); }
                    }
                }
                t0 = end;
                ++items;
            } else if (group < 2 && p.part <= 0 && (!PARTS || a.hs == 1)) {
                zero_tile<kRows>((bf16*)(group == 0 ? a.dK : a.dV) + p.b * a.kb + p.h * a.kh, a.kn, p.key0, a.n, row);
            }
            index = sched_next(sched, it, true, status);
            if (bar_any(1 + group, kRows, index < 0)) index = -1;            // (a whole warpgroup or none of it: it shares barriers)
            if (lane == 0) sched_taken(sched, it);
        }
        if (row == 0) bulk_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == Dkv::kMma) { cta_teardown_warp(); tmem_dealloc(tm, Dkv::kTmem); }
    if (warp < 4 * kGroups && !cta_gave_up())
        redo_noted(s_redo[warp], [&](uint32_t code) { return a.redo + (size_t)code * 4 + warp % 4; }, [&](uint32_t code, int k) {
            const KeyItem p = item((int)(code / 2));
            const int which = (int)(code % 2), r = warp % 4 * 32 + k, j = p.key0 + r;
            if (!key_tainted<bf16>(a, p.b, p.h, j, p.len, p.stop)) return;
            const KeyRow key = redo_dkv_row<bf16>(a, p.b, p.h, j, p.len, PARTS && p.part == 0 && r < a.sinks ? p.stop : p.len);
            const float2 v = which ? key.dv : key.dk;
            float* sum = PARTS ? sum_place(p, which, r) : nullptr;
            if (sum != nullptr) st2(sum + 2 * lane, v);
            else st2((bf16*)(which ? a.dV : a.dK) + p.b * a.kb + (PARTS ? p.h / a.hs : p.h) * a.kh + j * a.kn + 2 * lane, v);
        });
}

// The status word, in front of a kernel whose CTAs take over items: any item that has not been started may be taken over, the first one too, so
// that none of its CTAs is sure to clear the word, nor to do so before another may write it.
__global__ void win_clear_kernel(int* status) {
    pdl_sync();
    *status = 0;
}
void clear_status(int* status, cudaStream_t s) {
    prof_begin("win_clear_kernel", s);
    launch_pdl(win_clear_kernel, dim3(1), dim3(1), 0, s, status);
    prof_end(s);
}
ItemMap item_map(const WinArgs& a, int heads) {
    ItemMap m;
    m.tiles.set((uint32_t)((a.n + kRows - 1) / kRows));
    m.heads.set((uint32_t)heads);
    m.parts.set((uint32_t)(a.parts > 0 ? a.parts : 1));
    return m;
}
bool map_q(const WinArgs& a, CUtensorMap* m, const void* p, int rows) { return tc_map_rows(m, p, a.B, a.H, a.n, a.qb, a.qh, a.qn, rows); }
bool map_k(const WinArgs& a, CUtensorMap* m, const void* p, int rows) { return tc_map_rows(m, p, a.B, a.Hkv, a.n, a.kb, a.kh, a.kn, rows); }

}  // namespace

cudaError_t tc_window_fwd(const WinArgs& a, int* status, cudaStream_t s) {
    CUtensorMap mQ, mK, mV, mO;
    if (!map_q(a, &mQ, a.Q, 128) || !map_k(a, &mK, a.K, 128) || !map_k(a, &mV, a.V, 128) || !map_q(a, &mO, a.out, 128)) return cudaErrorInvalidValue;
    const unsigned items = (unsigned)((a.n + kRows - 1) / kRows) * a.B * a.H;
    const bool takes = items > 148u * Fwd::kPerSm;
    const auto fwd = takes ? tc_win_fwd_kernel<true> : tc_win_fwd_kernel<false>;
    PSK_TRY(set_smem(fwd, Fwd::bytes));
    if (takes) clear_status(status, s);
    prof_begin("tc_win_fwd_kernel", s);
    launch_pdl(fwd, dim3(items), dim3(Fwd::kThreads), Fwd::bytes, s, mQ, mK, mV, mO, a, item_map(a, a.H), status);
    prof_end(s);
    return cudaGetLastError();
}

cudaError_t tc_window_bwd(const WinArgs& a, const WinArgs& k, int* status, cudaStream_t s) {
    const unsigned tiles = (unsigned)((a.n + kRows - 1) / kRows);
    {
        CUtensorMap mQ, mG, mO, mK, mV, mDq;
        if (!map_q(a, &mQ, a.Q, 128) || !map_q(a, &mG, a.dO, 128) || !map_q(a, &mO, a.O, 128) || !map_k(a, &mK, a.K, 64) || !map_k(a, &mV, a.V, 64) || !map_q(a, &mDq, a.dQ, 128))
            return cudaErrorInvalidValue;
        const unsigned items = tiles * a.B * a.H;
        const bool takes = items > 148u;
        const auto dq = takes ? tc_win_dq_kernel<true> : tc_win_dq_kernel<false>;
        PSK_TRY(set_smem(dq, Dq::bytes));
        if (takes) clear_status(status, s);
        prof_begin("tc_win_dq_kernel", s);
        launch_pdl(dq, dim3(items), dim3(Dq::kThreads), Dq::bytes, s, mQ, mG, mO, mK, mV, mDq, a, item_map(a, a.H), status);
        prof_end(s);
    }
    CUtensorMap mK, mV, mQ, mG, mDk, mDv;
    if (!map_k(a, &mK, a.K, 128) || !map_k(a, &mV, a.V, 128) || !map_q(a, &mQ, a.Q, 64) || !map_q(a, &mG, a.dO, 64) || !map_k(a, &mDk, a.dK, 128) ||
        !map_k(a, &mDv, a.dV, 128))
        return cudaErrorInvalidValue;
    const auto dkv = k.parts > 0 || k.hs > 1 ? tc_win_dkv_kernel<true> : tc_win_dkv_kernel<false>;
    PSK_TRY(set_smem(dkv, Dkv::bytes));
    prof_begin("tc_win_dkv_kernel", s);
    launch_pdl(dkv, dim3((tiles + k.parts) * k.B * k.Hkv), dim3(Dkv::kThreads), Dkv::bytes, s, mK, mV, mQ, mG, mDk, mDv, k, item_map(k, k.Hkv), status);
    prof_end(s);
    return cudaGetLastError();
}

}  // namespace win
}  // namespace psk

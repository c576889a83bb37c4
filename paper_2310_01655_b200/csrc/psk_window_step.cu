// The cache of sliding-window attention, and the attention of one new token on it.
// A sequence's cache has `sinks + window` slots per key head: position p < sinks lies in slot p, a later one in slot
// sinks + (p - sinks) mod window.  After position t has been written, the slots below min(t + 1, sinks + window) hold exactly the
// positions that row t sees (the ring holds the last `window` of those behind the sinks, and softmax does not ask for
// their order), so that a sequence of any length keeps a state of fixed size, as psk_decode_step's.
#include "packed.cuh"
#include "psk_window.cuh"

namespace psk {
namespace win {
namespace {

__device__ __forceinline__ int slot_of(int p, int window, int sinks) { return p < sinks ? p : sinks + (p - sinks) % window; }

// ---------------------------------------------------------------------------
// Cache behind a prompt: one slot of one key head to 8 (bf16) or 16 (fp32) lanes, 16 bytes each.  Slots that no position of the
// sequence has are left as they are.  Bound: memory.
// ---------------------------------------------------------------------------
struct FillArgs {
    const void *K, *V;
    void *Kc, *Vc;
    const int32_t* lengths;
    int B, Hkv, n, window, sinks;
    int64_t kb, kh, kn, total;        // total: B Hkv slots
};

template <typename T>
__global__ void __launch_bounds__(256)
win_fill_kernel(const __grid_constant__ FillArgs a) {
    constexpr int L = 64 * sizeof(T) / 16, V = 16 / sizeof(T);
    pdl_sync();
    const int64_t slots = (int64_t)a.sinks + a.window, e = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    if (e >= a.total) return;
    const int64_t bh = e / slots, slot = e - bh * slots;
    const int b = (int)(bh / a.Hkv), h = (int)(bh % a.Hkv);
    int len = a.n;
    if (a.lengths != nullptr) { const int l = a.lengths[b]; len = l < 0 ? 0 : (l < a.n ? l : a.n); }
    int64_t p = slot;
    if (slot >= a.sinks) {
        // the last position whose slot this is
        const int64_t r = slot - a.sinks, last = (int64_t)len - 1 - a.sinks;
        if (r > last) return;
        p = a.sinks + r + (last - r) / a.window * a.window;
    }
    if (p >= len) return;
    const int c = threadIdx.x % L * V;
    const int64_t from = b * a.kb + h * a.kh + p * a.kn + c, to = e * 64 + c;
    const uint4 k = *reinterpret_cast<const uint4*>((const T*)a.K + from), v = *reinterpret_cast<const uint4*>((const T*)a.V + from);
    *reinterpret_cast<uint4*>((T*)a.Kc + to) = k;
    *reinterpret_cast<uint4*>((T*)a.Vc + to) = v;
}

// ---------------------------------------------------------------------------
// One new token, fp32 caches.  A cluster of CL CTAs has the NG query heads (at most 8) of one key head and sequence; each CTA has a
// stretch of the slots, each L = 16 lanes of a warp a slot at a time (16 bytes of a key and of a value per
// lane), U slots in flight, with a running maximum, sum and output per query head in registers (packed pairs).
// They are joined inside a warp by shuffles, inside a CTA through shared memory, and over the cluster in the first CTA's memory.
// The new key and value are read from the arguments, not from the cache: nobody waits for the slot to be written.
// Bound: reading the cache once; with few sequences, latency.
// ---------------------------------------------------------------------------
struct StepArgs {
    const void *q, *k, *v;
    void *Kc, *Vc, *o;
    const int32_t* positions;
    int H, Hkv, G, parts, window, sinks;      // parts: groups of query heads per key head
    float c;
};
constexpr int kStepThreads = 256, kStepWarps = kStepThreads / 32;

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ void unpack(const uint4& u, f2 (&f)[2]) {
    f[0] = pack2(u.x, u.y);
    f[1] = pack2(u.z, u.w);
}

// The warps of a CTA, then the CTAs of a cluster: maxima, sums and outputs of NG rows.
template <typename T, int NG, int CL, int WARPS>
__device__ __forceinline__ void join(const float (&s_m)[WARPS][NG], const float (&s_l)[WARPS][NG], const float (*s_o)[NG][64], float (&r_m)[CL][NG],
                                     float (&r_l)[CL][NG], float (&r_o)[CL][NG][64], int heads, int cr, T* o) {
    const int tid = threadIdx.x, threads = blockDim.x;
    __syncthreads();
    if (CL > 1) cluster_wait();                       // every CTA of the cluster has started
    for (int e = tid; e < heads * 64; e += threads) {
        const int g = e / 64, d = e % 64;
        float top = neg_inf(), lsum = 0.f, osum = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_m[w][g]);
        const float at = top == neg_inf() ? 0.f : top;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = exp2_approx(s_m[w][g] - at);
            lsum = fmaf(s_l[w][g], f, lsum);
            osum = fmaf(s_o[w][g][d], f, osum);
        }
        if (CL == 1) {
            stf(o + e, osum / lsum);
        } else {                                      // into the first CTA's memory
            auto put = [&](const float* mine, float v) {
                unsigned dst;
                asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(dst) : "r"((unsigned)__cvta_generic_to_shared(mine)));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(v) : "memory");
            };
            put(&r_o[cr][g][d], osum);
            if (d == 0) { put(&r_m[cr][g], top); put(&r_l[cr][g], lsum); }
        }
    }
    if (CL == 1) return;
    cluster_arrive();
    if (cr != 0) return;                              // nobody reads this CTA's memory
    cluster_wait();
    for (int e = tid; e < heads * 64; e += threads) {
        const int g = e / 64, d = e % 64;
        float top = neg_inf(), lsum = 0.f, osum = 0.f;
#pragma unroll
        for (int r = 0; r < CL; ++r) top = fmaxf(top, r_m[r][g]);
        const float at = top == neg_inf() ? 0.f : top;
#pragma unroll
        for (int r = 0; r < CL; ++r) {
            const float f = exp2_approx(r_m[r][g] - at);
            lsum = fmaf(r_l[r][g], f, lsum);
            osum = fmaf(r_o[r][g][d], f, osum);
        }
        stf(o + e, osum / lsum);
    }
}

template <int NG, int CL>
__global__ void __launch_bounds__(kStepThreads)
win_step_kernel(const __grid_constant__ StepArgs a) {
    typedef float T;
    constexpr int V = 4, P = V / 2, L = 64 / V, Groups = kStepThreads / L, U = NG >= 8 ? 2 : 4;
    __shared__ float s_m[kStepWarps][NG], s_l[kStepWarps][NG];
    __shared__ __align__(16) float s_o[kStepWarps][NG][64];
    __shared__ float r_m[CL][NG], r_l[CL][NG];                      // used in the cluster's first CTA
    __shared__ __align__(16) float r_o[CL][NG][64];
    pdl_sync();
    const int cr = (int)(blockIdx.x % CL), unit = blockIdx.x / CL, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const int part = unit % a.parts, bk = unit / a.parts, b = bk / a.Hkv, hk = bk % a.Hkv;
    const int g0 = part * NG, heads = a.G - g0 < NG ? a.G - g0 : NG;          // (the last group of query heads may be smaller)
    const int pos = a.positions[b];
    T* o = (T*)a.o + ((int64_t)b * a.H + (int64_t)hk * a.G + g0) * 64;
    if (pos < 0) {                                                            // an idle place (the same for the whole cluster)
        if (cr == 0)
            for (int e = tid; e < heads * 64; e += kStepThreads) stf(o + e, 0.f);
        return;
    }
    if (CL > 1) cluster_arrive();
    const int64_t slots = (int64_t)a.sinks + a.window, base = (int64_t)bk * slots;
    const int mine = slot_of(pos, a.window, a.sinks), held = (int64_t)pos + 1 < slots ? pos + 1 : (int)slots;
    const int c = lane % L * V;
    const T *knew = (const T*)a.k + (int64_t)bk * 64 + c, *vnew = (const T*)a.v + (int64_t)bk * 64 + c;
    T *Kc = (T*)a.Kc + base * 64 + c, *Vc = (T*)a.Vc + base * 64 + c;
    if (cr == 0 && part == 0 && tid < L) {
        *reinterpret_cast<uint4*>(Kc + (int64_t)mine * 64) = *reinterpret_cast<const uint4*>(knew);
        *reinterpret_cast<uint4*>(Vc + (int64_t)mine * 64) = *reinterpret_cast<const uint4*>(vnew);
    }
    f2 q[NG][P], acc[NG][P];
    float m[NG], l[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (g < heads) u = *reinterpret_cast<const uint4*>((const T*)a.q + ((int64_t)b * a.H + (int64_t)hk * a.G + g0 + g) * 64 + c);
        unpack(u, q[g]);
        m[g] = neg_inf();
        l[g] = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) { q[g][i] = mul2(q[g][i], pack2(a.c, a.c)); acc[g][i] = 0ull; }
    }
    // this CTA's slots
    const int chunk = (int)(((int64_t)held + CL - 1) / CL), first = (int64_t)cr * chunk < held ? cr * chunk : held;
    const int last = held - first < chunk ? held : first + chunk;
    const int group = tid / L;
    for (int64_t s0 = first; s0 < last; s0 += Groups * U) {
        uint4 ku[U], vu[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t s = s0 + u * Groups + group;
            const bool is_new = s == mine;
            ku[u] = vu[u] = make_uint4(0, 0, 0, 0);
            if (s < last) {
                ku[u] = *reinterpret_cast<const uint4*>(is_new ? knew : Kc + s * 64);
                vu[u] = *reinterpret_cast<const uint4*>(is_new ? vnew : Vc + s * 64);
            }
        }
        float sc[U][NG];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f2 kf[P];
            unpack(ku[u], kf);
            const bool in = s0 + u * Groups + group < last;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                f2 d = mul2(q[g][0], kf[0]);
#pragma unroll
                for (int i = 1; i < P; ++i) d = fma2(q[g][i], kf[i], d);
                float s = lo2(d) + hi2(d);
#pragma unroll
                for (int x = 1; x < L; x <<= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
                sc[u][g] = in ? s : neg_inf();
            }
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float top = m[g];
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, sc[u][g]);
            const float at = top == neg_inf() ? 0.f : top, alpha = exp2_approx(m[g] - at);
            m[g] = top;
            l[g] *= alpha;
#pragma unroll
            for (int i = 0; i < P; ++i) acc[g][i] = mul2(acc[g][i], pack2(alpha, alpha));
#pragma unroll
            for (int u = 0; u < U; ++u) { sc[u][g] = exp2_approx(sc[u][g] - at); l[g] += sc[u][g]; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f2 vf[P];
            unpack(vu[u], vf);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const f2 p2 = pack2(sc[u][g], sc[u][g]);
#pragma unroll
                for (int i = 0; i < P; ++i) acc[g][i] = fma2(p2, vf[i], acc[g][i]);
            }
        }
    }
    // the slots side by side in a warp
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        float top = m[g];
#pragma unroll
        for (int x = L; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        const float at = top == neg_inf() ? 0.f : top, alpha = exp2_approx(m[g] - at);
        l[g] *= alpha;
#pragma unroll
        for (int x = L; x < 32; x <<= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], x);
        float f[V];
#pragma unroll
        for (int i = 0; i < P; ++i) { f[2 * i] = lo2(acc[g][i]) * alpha; f[2 * i + 1] = hi2(acc[g][i]) * alpha; }
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int x = L; x < 32; x <<= 1) f[i] += __shfl_xor_sync(0xffffffffu, f[i], x);
        if (lane < L) {
#pragma unroll
            for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(&s_o[warp][g][c + i]) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
            if (lane == 0) { s_m[warp][g] = top; s_l[warp][g] = l[g]; }
        }
    }
    join<T, NG, CL, kStepWarps>(s_m, s_l, s_o, r_m, r_l, r_o, heads, cr, o);
}

// ---------------------------------------------------------------------------
// The same for bf16 caches with products on the warps' matrix instructions (16 x 8 x 16): up to 16 query heads are the rows of one
// operand, 16 slots a strip.  On the CUDA cores the products alone took more issue slots than the cache takes time to arrive
// (64 sequences, 4 key heads with 4 query heads each, 4100 slots: 238 us).  A weight is given to the second product as hi + lo,
// two bf16 terms, so that it keeps 2^-17.  Every warp has strips of its own in a ring of its own, filled by
// asynchronous copies (zeros for slots that are not held), and waits for nobody else until the join.
// Bound: reading the cache once.
// ---------------------------------------------------------------------------
constexpr int kStrip = 16, kStripBytes = kStrip * 256, kRing = 3;

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&v)[4], unsigned addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&v)[4], unsigned addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int CL, int WARPS, bool WIDE>          // WIDE: more than 8 query heads
__global__ void __launch_bounds__(32 * WARPS)
win_step_mma_kernel(const __grid_constant__ StepArgs a) {
    constexpr int kMmaWarps = WARPS, kMmaThreads = 32 * WARPS, NG = WIDE ? 16 : 8, RS = WIDE ? 2 : 1;             // rows of the operand in use; of them in a thread
    extern __shared__ __align__(128) uint8_t ring[];                 // [warp][kRing][K 16 x 128 B, V 16 x 128 B], chunks of a row swizzled; then outputs
    __shared__ float s_m[kMmaWarps][NG], s_l[kMmaWarps][NG];
    __shared__ float r_m[CL][NG], r_l[CL][NG];
    __shared__ __align__(16) float r_o[CL][NG][64];                  // used in the cluster's first CTA
    pdl_sync();
    const int cr = (int)(blockIdx.x % CL), unit = blockIdx.x / CL, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const int part = unit % a.parts, bk = unit / a.parts, b = bk / a.Hkv, hk = bk % a.Hkv;
    const int g0 = part * NG, heads = a.G - g0 < NG ? a.G - g0 : NG;
    const int pos = a.positions[b];
    const int64_t head0 = (int64_t)b * a.H + (int64_t)hk * a.G + g0;
    bf16* o = (bf16*)a.o + head0 * 64;
    if (pos < 0) {                                                   // an idle place (the same for the whole cluster)
        if (cr == 0)
            for (int e = tid; e < heads * 64; e += kMmaThreads) stf(o + e, 0.f);
        return;
    }
    if (CL > 1) cluster_arrive();
    const int64_t slots = (int64_t)a.sinks + a.window;
    const int mine = slot_of(pos, a.window, a.sinks), held = (int64_t)pos + 1 < slots ? pos + 1 : (int)slots;
    const bf16 *knew = (const bf16*)a.k + (int64_t)bk * 64, *vnew = (const bf16*)a.v + (int64_t)bk * 64;
    bf16 *Kc = (bf16*)a.Kc + bk * slots * 64, *Vc = (bf16*)a.Vc + bk * slots * 64;
    if (cr == 0 && part == 0 && tid < 16) {
        const int c = tid % 8 * 8;
        if (tid < 8) *reinterpret_cast<uint4*>(Kc + (int64_t)mine * 64 + c) = *reinterpret_cast<const uint4*>(knew + c);
        else *reinterpret_cast<uint4*>(Vc + (int64_t)mine * 64 + c) = *reinterpret_cast<const uint4*>(vnew + c);
    }
    // this CTA's strips, dealt to its warps in turn
    const int strips = (held - 1) / kStrip + 1, each = (strips + CL - 1) / CL;
    const int first = cr * each < strips ? cr * each : strips, last = strips - first < each ? strips : first + each;
    uint8_t* buf = ring + warp * kRing * kStripBytes;
    const unsigned buf_s = (unsigned)__cvta_generic_to_shared(buf);
    const int lr = lane / 8, lc = lane % 8;                          // this lane copies rows lr, lr + 4, ..., 16-byte chunk lc
    auto request = [&](int strip, int stage) {
        if (strip < last) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = lr + 4 * k;
                const int64_t s = (int64_t)strip * kStrip + r;
                const unsigned dst = buf_s + stage * kStripBytes + r * 128 + ((lc ^ (r & 7)) << 4);
                const bool in = s < held, is_new = s == mine;
                const bf16 *ks = is_new || !in ? knew : Kc + s * 64, *vs = is_new || !in ? vnew : Vc + s * 64;
                const int bytes = in ? 16 : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(ks + lc * 8), "r"(bytes) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + kStrip * 128), "l"(vs + lc * 8), "r"(bytes) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kRing - 1; ++k) request(first + warp + k * kMmaWarps, k);
    // Q as the first operand: rows lane / 4 and lane / 4 + 8, columns 2 (lane % 4) and 8 on
    uint32_t q[4][4];
    const int g = lane / 4, cq = lane % 4 * 2;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = g + (e & 1) * 8;
            q[kk][e] = r < heads ? *reinterpret_cast<const uint32_t*>((const bf16*)a.q + (head0 + r) * 64 + kk * 16 + (e >> 1) * 8 + cq) : 0u;
        }
    float m[RS], l[RS], acc[8][4];
#pragma unroll
    for (int r = 0; r < RS; ++r) { m[r] = neg_inf(); l[r] = 0.f; }
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
    int stage = 0;
#pragma unroll 1
    for (int strip = first + warp; strip < last; strip += kMmaWarps) {
        request(strip + (kRing - 1) * kMmaWarps, stage == 0 ? kRing - 1 : stage - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
        __syncwarp();
        const unsigned base = buf_s + stage * kStripBytes;
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        const int kr = lane / 16 * 8 + lane % 8;                     // the row of K whose chunk this lane points at
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            uint32_t kf[4];
            ldsm4(kf, base + kr * 128 + (((2 * kk + lane / 8 % 2) ^ (kr & 7)) << 4));
            mma16816(s[0], q[kk], kf[0], kf[1]);
            mma16816(s[1], q[kk], kf[2], kf[3]);
        }
        const int rest = held - strip * kStrip;                      // slots of this strip and behind it
        float alpha[RS];
        uint32_t hi[4] = {0, 0, 0, 0}, lo[4] = {0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < RS; ++r) {
            float p[4], top = m[r];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = s[e / 2][2 * r + e % 2] * a.c;
                if (rest < kStrip && e / 2 * 8 + cq + e % 2 >= rest) p[e] = neg_inf();
                top = fmaxf(top, p[e]);
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float at = top == neg_inf() ? 0.f : top;
            alpha[r] = exp2_approx(m[r] - at);
            m[r] = top;
            l[r] *= alpha[r];
#pragma unroll
            for (int e = 0; e < 4; ++e) { p[e] = exp2_approx(p[e] - at); l[r] += p[e]; }
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const uint32_t h = pack_pair(p[e], p[e + 1]);
                hi[e + r] = h;
                lo[e + r] = pack_pair(p[e] - __uint_as_float(h << 16), p[e + 1] - __uint_as_float(h & 0xffff0000u));
            }
        }
        bool same = true;
#pragma unroll
        for (int r = 0; r < RS; ++r) same = same && alpha[r] == 1.f;
        if (!__all_sync(0xffffffffu, same))
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 2 * RS; ++e) acc[n][e] *= alpha[e / 2];
        const int vr = lane % 16;
#pragma unroll
        for (int n = 0; n < 8; n += 2) {
            uint32_t vf[4];
            ldsm4_trans(vf, base + kStrip * 128 + vr * 128 + (((n + lane / 16) ^ (vr & 7)) << 4));
            mma16816(acc[n], hi, vf[0], vf[1]);
            mma16816(acc[n + 1], hi, vf[2], vf[3]);
            mma16816(acc[n], lo, vf[0], vf[1]);
            mma16816(acc[n + 1], lo, vf[2], vf[3]);
        }
        __syncwarp();                                                // everyone has read the stage that is asked for next
        stage = stage + 1 == kRing ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                                                 // the rings take the outputs
    float(*s_o)[NG][64] = reinterpret_cast<float(*)[NG][64]>(ring);
#pragma unroll
    for (int r = 0; r < RS; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        if (lane % 4 == 0) { s_m[warp][g + 8 * r] = m[r]; s_l[warp][g + 8 * r] = l[r]; }
#pragma unroll
        for (int n = 0; n < 8; ++n) *reinterpret_cast<float2*>(&s_o[warp][g + 8 * r][8 * n + cq]) = make_float2(acc[n][2 * r], acc[n][2 * r + 1]);
    }
    join<bf16, NG, CL, kMmaWarps>(s_m, s_l, s_o, r_m, r_l, r_o, heads, cr, o);
}

template <int CL, typename Kern>
cudaError_t launch_cl(Kern kern, const StepArgs& a, int64_t units, int threads, int smem, cudaStream_t s) {
    if (smem > 0) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * CL));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CL; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    prof_begin("win_step_kernel", s);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a);
    prof_end(s);
    return e == cudaSuccess ? cudaGetLastError() : e;
}
// CTAs per key head: enough for `want` in all, but a stretch of the cache of `least` slots at least (where the caches are full)
int cluster_size(const StepArgs& a, int64_t units, int want, int least) {
    const int64_t slots = (int64_t)a.sinks + a.window;
    int cl = 1;
    while (cl < 8 && units * cl < want && slots / (2 * cl) >= least) cl *= 2;
    return cl;
}
template <int NG>
cudaError_t launch_ng(const StepArgs& a, int64_t units, cudaStream_t s) {
    // (fp32, us with stretches of 32 / 64 slots at least; 12 heads x 501 slots: 4.3 / 5.7)
    switch (cluster_size(a, units, 300, 32)) {
        case 1: return launch_cl<1>(win_step_kernel<NG, 1>, a, units, kStepThreads, 0, s);
        case 2: return launch_cl<2>(win_step_kernel<NG, 2>, a, units, kStepThreads, 0, s);
        case 4: return launch_cl<4>(win_step_kernel<NG, 4>, a, units, kStepThreads, 0, s);
        default: return launch_cl<8>(win_step_kernel<NG, 8>, a, units, kStepThreads, 0, s);
    }
}
cudaError_t launch_f32(StepArgs a, int64_t keyheads, cudaStream_t s) {
    a.parts = (a.G + 7) / 8;
    if (a.G == 1) return launch_ng<1>(a, keyheads, s);
    if (a.G == 2) return launch_ng<2>(a, keyheads, s);
    if (a.G <= 4) return launch_ng<4>(a, keyheads, s);
    return launch_ng<8>(a, keyheads * a.parts, s);
}
template <int CL, bool WIDE>
cudaError_t launch_warps(const StepArgs& a, int64_t units, cudaStream_t s) {
    // A strip is a chain of a thousand cycles: where a CTA has its SM to itself and eight strips for each warp, eight warps instead of four
    // (12 heads x 8196 slots: 11.4 -> 10.1 us; 128 heads x 64: 2.7 with four, 3.0 with eight).
    if (units * CL <= 148 && ((int64_t)a.sinks + a.window) / CL >= 512) return launch_cl<CL>(win_step_mma_kernel<CL, 8, WIDE>, a, units, 256, 8 * kRing * kStripBytes, s);
    return launch_cl<CL>(win_step_mma_kernel<CL, 4, WIDE>, a, units, 128, 4 * kRing * kStripBytes, s);
}
template <bool WIDE>
cudaError_t launch_mma(const StepArgs& a, int64_t units, cudaStream_t s) {
    // (us with 250 / 600 CTAs wanted; 64 sequences x 4 key heads x 4100 slots: 44.5 / 51.7, 8 x 12 x 1028: 8.6 / 12.6, 32 x 12 x 512: 11.8 / 15.6)
    switch (cluster_size(a, units, 250, 128)) {
        case 1: return launch_warps<1, WIDE>(a, units, s);
        case 2: return launch_warps<2, WIDE>(a, units, s);
        case 4: return launch_warps<4, WIDE>(a, units, s);
        default: return launch_warps<8, WIDE>(a, units, s);
    }
}
cudaError_t launch_bf16(StepArgs a, int64_t keyheads, cudaStream_t s) {
    a.parts = (a.G + 15) / 16;
    return a.G <= 8 ? launch_mma<false>(a, keyheads, s) : launch_mma<true>(a, keyheads * a.parts, s);
}

// slots whose byte offsets and grid sizes stay in range
bool cache_ok(const psk_window_shape* sh) {
    const int64_t slots = (int64_t)sh->sinks + sh->window;
    return slots < (int64_t)1 << 31 && (int64_t)sh->B * sh->Hkv < ((int64_t)1 << 40) / slots;
}

}  // namespace
}  // namespace win
}  // namespace psk

using namespace psk;
using namespace psk::win;

extern "C" {

size_t psk_window_cache_bytes(const psk_window_shape* shape) {
    if (check_common(shape) != PSK_OK || !cache_ok(shape)) return 0;
    return (size_t)shape->B * shape->Hkv * ((size_t)shape->sinks + shape->window) * 64 * (shape->dtype == PSK_F32 ? 4 : 2);
}

int psk_window_cache_fill(const psk_window_shape* shape, const void* K, const void* V, const int32_t* lengths, void* Kc, void* Vc, void* stream) {
    const int st = check_rows(shape);
    if (st != PSK_OK) return st;
    if (!cache_ok(shape)) return PSK_ERR_SHAPE;
    if (!K || !V || !Kc || !Vc) return PSK_ERR_INVALID_ARG;
    for (const void* p : {K, V, (const void*)Kc, (const void*)Vc})
        if (!aligned16(p)) return PSK_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(lengths) & 3u) return PSK_ERR_ALIGN;
    const WinArgs w = args_of(shape);
    FillArgs a{K, V, Kc, Vc, lengths, w.B, w.Hkv, w.n, w.window, w.sinks, w.kb, w.kh, w.kn, (int64_t)w.B * w.Hkv * ((int64_t)w.sinks + w.window)};
    const int per = shape->dtype == PSK_F32 ? 16 : 32;
    const int64_t grid = (a.total + per - 1) / per;
    if (grid >= (int64_t)1 << 31) return PSK_ERR_SHAPE;
    CountLaunches count;
    cudaStream_t s = (cudaStream_t)stream;
    prof_begin("win_fill_kernel", s);
    if (shape->dtype == PSK_F32) launch_pdl(win_fill_kernel<float>, dim3((unsigned)grid), dim3(256), 0, s, a);
    else launch_pdl(win_fill_kernel<bf16>, dim3((unsigned)grid), dim3(256), 0, s, a);
    prof_end(s);
    return cudaGetLastError() == cudaSuccess ? PSK_OK : PSK_ERR_CUDA;
}

int psk_window_decode_step(const psk_window_shape* shape, const void* q, const void* k, const void* v, const int32_t* positions, void* Kc, void* Vc,
                           void* o, void* stream) {
    const int st = check_common(shape);
    if (st != PSK_OK) return st;
    if (!cache_ok(shape) || (int64_t)shape->B * shape->H >= (int64_t)1 << 28) return PSK_ERR_SHAPE;
    if (!q || !k || !v || !positions || !Kc || !Vc || !o) return PSK_ERR_INVALID_ARG;
    for (const void* p : {q, k, v, (const void*)Kc, (const void*)Vc, (const void*)o})
        if (!aligned16(p)) return PSK_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(positions) & 3u) return PSK_ERR_ALIGN;
    StepArgs a{q, k, v, Kc, Vc, o, positions, shape->H, shape->Hkv, shape->H / shape->Hkv, 1, shape->window, shape->sinks, shape->scale * kLog2e};
    const int64_t keyheads = (int64_t)shape->B * shape->Hkv;
    CountLaunches count;
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = shape->dtype == PSK_F32 ? launch_f32(a, keyheads, s) : launch_bf16(a, keyheads, s);
    return e == cudaSuccess ? PSK_OK : PSK_ERR_CUDA;
}

}  // extern "C"

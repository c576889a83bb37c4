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
// One new token.  A cluster of CL CTAs has the NG query heads (at most 8) of one key head and sequence; each CTA has a
// stretch of the slots, each L = 8 (bf16) or 16 (fp32) lanes of a warp a slot at a time (16 bytes of a key and of a value per
// lane), U slots in flight, with a running maximum, sum and output per query head in registers (fp32, packed pairs).
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

template <typename T> __device__ __forceinline__ void unpack(const uint4& u, f2 (&f)[8 / sizeof(T)]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack2(w[i] << 16, w[i] & 0xffff0000u);
    } else {
        f[0] = pack2(w[0], w[1]);
        f[1] = pack2(w[2], w[3]);
    }
}

template <typename T, int NG, int CL>
__global__ void __launch_bounds__(kStepThreads)
win_step_kernel(const __grid_constant__ StepArgs a) {
    constexpr int V = 16 / sizeof(T), P = V / 2, L = 64 / V, Groups = kStepThreads / L, U = NG >= 8 ? 2 : 4;
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
        unpack<T>(u, q[g]);
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
            unpack<T>(ku[u], kf);
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
            unpack<T>(vu[u], vf);
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
    __syncthreads();
    if (CL > 1) cluster_wait();                       // every CTA of the cluster has started
    // the warps of this CTA, into the first CTA's memory
    for (int e = tid; e < NG * 64; e += kStepThreads) {
        const int g = e / 64, d = e % 64;
        float top = neg_inf(), lsum = 0.f, osum = 0.f;
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) top = fmaxf(top, s_m[w][g]);
        const float at = top == neg_inf() ? 0.f : top;
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) {
            const float f = exp2_approx(s_m[w][g] - at);
            lsum = fmaf(s_l[w][g], f, lsum);
            osum = fmaf(s_o[w][g][d], f, osum);
        }
        if (CL == 1) {
            if (g < heads) stf(o + e, osum / lsum);
        } else {
            auto put = [&](const float* at_mine, float v) {
                unsigned dst;
                asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(dst) : "r"((unsigned)__cvta_generic_to_shared(at_mine)));
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
    for (int e = tid; e < heads * 64; e += kStepThreads) {
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

template <typename T, int NG, int CL>
cudaError_t launch_cl(const StepArgs& a, int64_t units, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units * CL));
    cfg.blockDim = dim3(kStepThreads);
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CL; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    prof_begin("win_step_kernel", s);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, win_step_kernel<T, NG, CL>, a);
    prof_end(s);
    return e == cudaSuccess ? cudaGetLastError() : e;
}
template <typename T, int NG>
cudaError_t launch_ng(const StepArgs& a, int64_t units, cudaStream_t s) {
    // CTAs per key head: enough that all SMs have two, but a stretch of the cache of 128 slots at least (where the caches are full)
    const int64_t slots = (int64_t)a.sinks + a.window;
    int cl = 1;
    while (cl < 8 && units * cl < 296 && slots / cl >= 256) cl *= 2;
    switch (cl) {
        case 1: return launch_cl<T, NG, 1>(a, units, s);
        case 2: return launch_cl<T, NG, 2>(a, units, s);
        case 4: return launch_cl<T, NG, 4>(a, units, s);
        default: return launch_cl<T, NG, 8>(a, units, s);
    }
}
template <typename T>
cudaError_t launch_step(StepArgs a, int64_t keyheads, cudaStream_t s) {
    if (a.G == 1) { a.parts = 1; return launch_ng<T, 1>(a, keyheads, s); }
    if (a.G == 2) { a.parts = 1; return launch_ng<T, 2>(a, keyheads, s); }
    if (a.G <= 4) { a.parts = 1; return launch_ng<T, 4>(a, keyheads, s); }
    a.parts = (a.G + 7) / 8;
    return launch_ng<T, 8>(a, keyheads * a.parts, s);
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
    cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = shape->dtype == PSK_F32 ? launch_step<float>(a, keyheads, s) : launch_step<bf16>(a, keyheads, s);
    return e == cudaSuccess ? PSK_OK : PSK_ERR_CUDA;
}

}  // extern "C"

// Group norm with an activation, channels last: what the forward and the backward pass share.
#pragma once

#include "ogq_act8.cuh"
#include "ogq_internal.h"

namespace ogq {

// A tile of the streaming kernels: `tx` vectors of V channels side by side, `ty` pixels at a time, `px` pixels a thread, all
// of one sample.  Each thread stays on its channels.
struct GnTiles {
    int64_t P, C, G;
    int cv;         // vectors of channels of a pixel
    int tx, ty, px;
    int ctiles;     // tiles side by side
    int chunks;     // tiles of pixels of one sample
    int64_t ctas;
};

constexpr int kGnMaxPx = 64;                 // pixels a thread, at most: sums in fp32 stay short
constexpr int kGnMinChunk = 16;              // pixels of a chunk whose sums are kept, at least: partial sums stay few

// Tiles for a kernel of which `wave` CTAs run at a time: whole waves, as near as the sizes allow (25.7 M bf16 values, moments: 800
// CTAs on 592 places took 19 us, 576 15), of at least `least` pixels a chunk and two a thread.
inline GnTiles gn_tiles(int64_t N, int64_t P, int64_t C, int64_t G, int V, int64_t wave, int least)
{
    GnTiles t;
    t.P = P; t.C = C; t.G = G;
    t.cv = (int)(C / V);
    t.tx = t.cv < kThreads ? t.cv : kThreads;
    t.ty = kThreads / t.tx;
    t.ctiles = (int)(((int64_t)t.cv + t.tx - 1) / t.tx);
    const int64_t units = (P + t.ty - 1) / t.ty, tasks = N * t.ctiles;  // pixels a thread of a sample, samples and tiles across
    int64_t px = kGnMaxPx;
    if (tasks > 0) {
        for (int64_t waves = 1; waves <= 16; ++waves) {
            const int64_t chunks = wave * waves / tasks;
            if (chunks == 0) continue;
            const int64_t q = (units + chunks - 1) / chunks;
            if (q <= kGnMaxPx) { px = q; break; }
        }
    }
    const int64_t lower = (least + t.ty - 1) / t.ty < 2 ? 2 : (least + t.ty - 1) / t.ty;
    t.px = (int)(px < lower ? lower : px);
    t.chunks = (int)((units + t.px - 1) / t.px);
    t.ctas = tasks * t.chunks;
    return t;
}

// CTAs of a kernel that run at a time, asked of the runtime at every launch (it depends on the instantiation and on the device).
template <class K>
inline int64_t gn_wave(K kernel, int sm_count)
{
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kThreads, 0) != cudaSuccess || n < 1) n = 1;
    return (int64_t)n * sm_count;
}

// Scratch: a pair per sample, chunk of pixels and channel, and a pair per sample and group.
struct GnWs {
    float2* part;  // [N][chunks][C]
    float2* sums;  // [N][G]
};
inline size_t gn_part_bytes(int64_t N, int64_t P, int64_t C)
{
    return (size_t)(N * ((P + kGnMinChunk - 1) / kGnMinChunk) * C) * sizeof(float2);
}
inline GnWs gn_ws(void* ws, int64_t N, int64_t G)
{
    GnWs w;
    w.sums = (float2*)ws;
    w.part = (float2*)((char*)ws + ((size_t)(N * G) * sizeof(float2) + 255) / 256 * 256);
    return w;
}

struct GnArgs {
    GnTiles t;
    const void* x;
    const void* dy;
    int8_t* codes;
    uint8_t* scales;
    void* out;
    const float* gamma;
    const float* beta;
    float* mean;
    float* rstd;
    float* dgamma;
    float* dbeta;
    float2* part;
    float2* sums;
    int64_t N;
    float eps;
    int act;
    uint32_t stream_id;
    PhiloxKeys keys;
};

inline GnArgs gn_args(const GroupNorm& p, const GnTiles& t)
{
    GnArgs a = {};
    const GnWs w = gn_ws(p.ws, p.N, p.G);
    a.t = t;
    a.x = p.x; a.dy = p.dy; a.codes = p.codes; a.scales = p.scales; a.out = p.out;
    a.gamma = p.gamma; a.beta = p.beta; a.mean = p.mean; a.rstd = p.rstd;
    a.dgamma = p.dgamma; a.dbeta = p.dbeta;
    a.part = w.part; a.sums = w.sums;
    a.N = p.N; a.eps = p.eps; a.act = p.act; a.stream_id = p.stream_id;
    a.keys = philox_round_keys((uint32_t)p.seed, (uint32_t)(p.seed >> 32));
    return a;
}

inline bool gn_aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// This thread's place: sample, chunk, and its pixels: the first one's row of the matrix [N P, C], how many (each ty rows on), channel c.
struct GnPlace {
    int64_t row;
    int64_t c;
    int n, chunk, tile, tx, ty, count;
    bool active;
};
template <int V>
__device__ __forceinline__ GnPlace gn_place(const GnTiles& t)
{
    GnPlace q;
    uint32_t nc = blockIdx.x;
    q.tile = 0;
    if (t.ctiles > 1) {
        nc = blockIdx.x / (uint32_t)t.ctiles;
        q.tile = (int)(blockIdx.x - nc * (uint32_t)t.ctiles);
    }
    q.n = (int)(nc / (uint32_t)t.chunks);
    q.chunk = (int)(nc - (uint32_t)q.n * (uint32_t)t.chunks);
    q.ty = (int)(threadIdx.x / (uint32_t)t.tx);
    q.tx = (int)threadIdx.x - q.ty * t.tx;
    const int64_t first = (int64_t)q.chunk * (t.ty * t.px) + q.ty;
    const uint32_t cv = (uint32_t)q.tile * (uint32_t)t.tx + (uint32_t)q.tx;  // the last tile's may lie past 2^31
    q.active = q.ty < t.ty && cv < (uint32_t)t.cv;
    q.c = (int64_t)cv * V;
    q.row = q.n * t.P + first;
    const int64_t left = t.P - first;
    q.count = left <= 0 ? 0 : left >= (int64_t)t.ty * t.px ? t.px : min(t.px, (int)((uint32_t)(left - 1) / (uint32_t)t.ty) + 1);
    return q;
}

// Calls fetch(i, r) and body(i, r) for pixels i = 0 ... count - 1; while B of them are worked on the next B are under way.  (All CTAs
// run at the same time here: without that they wait for memory together and compute together.)
template <class R, int B, class Fetch, class Body>
__device__ __forceinline__ void gn_pixels(int count, Fetch fetch, Body body)
{
    R r[2][B];
    const auto load = [&](int i, R (&t)[B]) {
#pragma unroll
        for (int k = 0; k < B; ++k)
            if (i + k < count) fetch(i + k, t[k]);
    };
    const auto work = [&](int i, const R (&t)[B]) {
#pragma unroll
        for (int k = 0; k < B; ++k)
            if (i + k < count) body(i + k, t[k]);
    };
    load(0, r[0]);
    for (int i = 0; i < count; i += 2 * B) {
        load(i + B, r[1]);
        work(i, r[0]);
        load(i + 2 * B, r[0]);
        work(i + B, r[1]);
    }
}

template <class E, int V>
__device__ __forceinline__ void gn_store(E* p, const float (&v)[V])
{
    if constexpr (V == 8) store8(p, v);
    else store1(p, v[0]);
}
// ACT < 0: chosen by `act` at run time (the kernels of single channels)
template <int ACT, bool ACCURATE>
__device__ __forceinline__ float gn_value(int act, float z)
{
    if constexpr (ACT >= 0) return act_value<ACT, ACCURATE>(z);
    switch (act) {
        case OGQ_ACT_RELU: return act_value<OGQ_ACT_RELU, ACCURATE>(z);
        case OGQ_ACT_SILU: return act_value<OGQ_ACT_SILU, ACCURATE>(z);
        case OGQ_ACT_GELU: return act_value<OGQ_ACT_GELU, ACCURATE>(z);
        default: return z;
    }
}
template <int ACT, bool ACCURATE>
__device__ __forceinline__ float gn_slope(int act, float z)
{
    if constexpr (ACT >= 0) return act_slope<ACT, ACCURATE>(z);
    switch (act) {
        case OGQ_ACT_RELU: return act_slope<OGQ_ACT_RELU, ACCURATE>(z);
        case OGQ_ACT_SILU: return act_slope<OGQ_ACT_SILU, ACCURATE>(z);
        case OGQ_ACT_GELU: return act_slope<OGQ_ACT_GELU, ACCURATE>(z);
        default: return 1.f;
    }
}

// V channels from c on of sample n: z = xh gamma + beta as a multiply-add of x - mean, a difference that is exact where x is near the mean.  (With the mean in the
// addend, beta - mean scale, z was off by 2^-24 |mean| rstd: a group of one value, rstd = 316, did not give beta, and the two passes could take different sides of ReLU.)
template <int V>
struct GnAffine {
    float mean[V], scale[V], shift[V];
    __device__ __forceinline__ void set(int j, float m, float rstd, float gamma, float beta)
    {
        mean[j] = m;
        scale[j] = __fmul_rn(rstd, gamma);
        shift[j] = beta;
    }
    __device__ __forceinline__ float centre(float x, int j) const { return __fsub_rn(x, mean[j]); }
    __device__ __forceinline__ float z(float centred, int j) const { return __fmaf_rn(centred, scale[j], shift[j]); }
};
// Calls f(j, mean, rstd, group) for V channels from c on of sample n.
template <int V, class F>
__device__ __forceinline__ void gn_channels(const GnArgs& a, int64_t n, int64_t c, F f)
{
    const int per = (int)(a.t.C / a.t.G);
    int g = (int)c / per;
    int left = (g + 1) * per - (int)c;  // channels until the next group
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (left == 0) { ++g; left = per; }
        --left;
        const int64_t at = n * a.t.G + g;
        f(j, a.mean[at], a.rstd[at], at);  // (from L1 where they are asked for again)
    }
}
template <int V>
__device__ __forceinline__ void gn_affine(const GnArgs& a, int64_t n, int64_t c, GnAffine<V>& f)
{
    gn_channels<V>(a, n, c, [&](int j, float mean, float rstd, int64_t) {
        f.set(j, mean, rstd, a.gamma ? a.gamma[c + j] : 1.f, a.beta ? a.beta[c + j] : 0.f);
    });
}
// dx = dz scale + (x - mean) slope + offset, from the group's means of gamma dz and gamma dz xh.
__device__ __forceinline__ void gn_gradient_terms(float2 means, float rstd, float& slope, float& offset)
{
    slope = -__fmul_rn(__fmul_rn(rstd, rstd), means.y);
    offset = -__fmul_rn(rstd, means.x);
}
// V elements as they lie in memory.
template <class E, int V> struct GnRaw { E e; };
template <class E> struct GnRaw<E, 8> { Raw8<E> e; };
// (volatile: the compiler otherwise moves a load that was asked for early back to where its value is needed)
__device__ __forceinline__ uint4 gn_load16(const void* p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <class E, int V>
__device__ __forceinline__ GnRaw<E, V> gn_fetch(const E* p)
{
    GnRaw<E, V> r;
    if constexpr (V == 8) {
        r.e.a = gn_load16(p);
        if constexpr (sizeof(E) == 4) r.e.b = gn_load16(p + 4);
    } else {
        r.e = *p;
    }
    return r;
}
template <class E, int V>
__device__ __forceinline__ void gn_open(const GnRaw<E, V>& r, float (&v)[V])
{
    if constexpr (V == 8) unpack8(r.e, v);
    else v[0] = load1(&r.e);
}
// The same of kept values.
template <int V> struct GnKept { int8_t c; uint32_t s; };
template <> struct GnKept<8> { uint2 c; uint32_t s; };
template <int V>
__device__ __forceinline__ GnKept<V> gn_fetch_kept(const int8_t* code, const uint8_t* scale)
{
    GnKept<V> r;
    if constexpr (V == 8) {
        asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(r.c.x), "=r"(r.c.y) : "l"(code));
        asm volatile("ld.global.u8 %0, [%1];" : "=r"(r.s) : "l"(scale));
    } else {
        r.c = *code;
        r.s = *scale;
    }
    return r;
}
template <int V>
__device__ __forceinline__ void gn_open(const GnKept<V>& r, float (&v)[V])
{
    if constexpr (V == 8) act8_values(r.c, act8_unit(r.s), v);
    else v[0] = (float)r.c * act8_unit(r.s);
}

}  // namespace ogq

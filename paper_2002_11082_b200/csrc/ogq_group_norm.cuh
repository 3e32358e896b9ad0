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

constexpr int kGnMinPx = 16, kGnMaxPx = 64;  // pixels a thread: sums in fp32 stay short, partial sums stay few
constexpr int kGnBatch = 4;                  // of them are loaded at once

inline GnTiles gn_tiles(int64_t N, int64_t P, int64_t C, int64_t G, int V, int sm_count)
{
    GnTiles t;
    t.P = P; t.C = C; t.G = G;
    t.cv = (int)(C / V);
    t.tx = t.cv < kThreads ? t.cv : kThreads;
    t.ty = kThreads / t.tx;
    t.ctiles = (t.cv + t.tx - 1) / t.tx;
    t.px = kGnMaxPx;
    for (;; t.px /= 2) {
        t.chunks = (int)((P + (int64_t)t.ty * t.px - 1) / ((int64_t)t.ty * t.px));
        t.ctas = N * t.chunks * t.ctiles;
        if (t.ctas >= (int64_t)sm_count * 4 || t.px == kGnMinPx) break;
    }
    return t;
}

// Scratch: a pair per sample, chunk of pixels and channel, and a pair per sample and group.
struct GnWs {
    float2* part;  // [N][chunks][C]
    float2* sums;  // [N][G]
};
inline size_t gn_part_bytes(int64_t N, int64_t P, int64_t C)
{
    const int64_t tx = C < kThreads ? C : kThreads, ty = kThreads / tx;  // single channels have the most chunks (vectors have larger ty)
    const int64_t chunks = (P + ty * kGnMinPx - 1) / (ty * kGnMinPx);
    return (size_t)(N * chunks * C) * sizeof(float2);
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

// This thread's place: sample, pixels first, first + ty, ... below last, first channel c (active: it has any).
struct GnPlace {
    int64_t n;
    int chunk, tx, ty;
    int64_t first, last, c;
    bool active;
};
template <int V>
__device__ __forceinline__ GnPlace gn_place(const GnTiles& t)
{
    GnPlace q;
    const int64_t b = blockIdx.x;
    const int64_t nc = b / t.ctiles;
    const int tile = (int)(b - nc * t.ctiles);
    q.n = nc / t.chunks;
    q.chunk = (int)(nc - q.n * t.chunks);
    q.ty = threadIdx.x / t.tx;
    q.tx = threadIdx.x - q.ty * t.tx;
    const int64_t begin = (int64_t)q.chunk * t.ty * t.px;
    q.first = begin + q.ty;
    q.last = begin + (int64_t)t.ty * t.px < t.P ? begin + (int64_t)t.ty * t.px : t.P;
    const int cv = tile * t.tx + q.tx;
    q.active = q.ty < t.ty && cv < t.cv;
    q.c = (int64_t)cv * V;
    return q;
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

// Parameters and statistics of V channels from c on, of sample n, and xh = (x - mean) rstd.  fp32 activations: the difference
// first, which is exact where x is near the mean.  16-bit ones: one multiply-add with mean rstd, off by 2^-24 |mean| rstd where
// their own rounding is 2^-9 or 2^-12 |x| rstd.
template <int V, bool ACCURATE>
struct GnChannels {
    float mean[V], rstd[V], gamma[V], beta[V];  // not ACCURATE: mean holds -mean rstd
    __device__ __forceinline__ void load(const GnArgs& a, int64_t n, int64_t c)
    {
        const int per = (int)(a.t.C / a.t.G);
        int g = (int)c / per;
        int left = (g + 1) * per - (int)c;  // channels until the next group
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (left == 0) { ++g; left = per; }
            --left;
            mean[j] = a.mean[n * a.t.G + g];
            rstd[j] = a.rstd[n * a.t.G + g];
            gamma[j] = a.gamma ? a.gamma[c + j] : 1.f;
            beta[j] = a.beta ? a.beta[c + j] : 0.f;
            if constexpr (!ACCURATE) mean[j] = __fmul_rn(-mean[j], rstd[j]);
        }
    }
    __device__ __forceinline__ float xh(float x, int j) const
    {
        if constexpr (ACCURATE) return __fmul_rn(__fsub_rn(x, mean[j]), rstd[j]);
        return __fmaf_rn(x, rstd[j], mean[j]);
    }
};

// z = xh gamma + beta of V channels, for the forward pass: one multiply-add more than the difference, or none.
template <int V, bool ACCURATE>
struct GnAffine {
    float mean[V], scale[V], shift[V];
    __device__ __forceinline__ void set(int j, float m, float rstd, float gamma, float beta)
    {
        mean[j] = m;
        scale[j] = __fmul_rn(rstd, gamma);
        shift[j] = ACCURATE ? beta : __fmaf_rn(-m, scale[j], beta);
    }
    __device__ __forceinline__ float z(float x, int j) const
    {
        return __fmaf_rn(ACCURATE ? __fsub_rn(x, mean[j]) : x, scale[j], shift[j]);
    }
};

// V elements as they lie in memory.
template <class E, int V> struct GnRaw { E e; };
template <class E> struct GnRaw<E, 8> { Raw8<E> e; };
template <class E, int V>
__device__ __forceinline__ GnRaw<E, V> gn_fetch(const E* p)
{
    GnRaw<E, V> r;
    if constexpr (V == 8) r.e = load_raw8(p);
    else r.e = *p;
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
__device__ __forceinline__ GnKept<V> gn_fetch_kept(const int8_t* codes, const uint8_t* scales, int64_t row, int64_t C, int64_t groups, int64_t c)
{
    GnKept<V> r;
    if constexpr (V == 8) r.c = *reinterpret_cast<const uint2*>(codes + row * C + c);
    else r.c = codes[row * C + c];
    r.s = scales[row * groups + c / kAct8Group];
    return r;
}
template <int V>
__device__ __forceinline__ void gn_open(const GnKept<V>& r, float (&v)[V])
{
    if constexpr (V == 8) act8_values(r.c, act8_unit(r.s), v);
    else v[0] = (float)r.c * act8_unit(r.s);
}

}  // namespace ogq

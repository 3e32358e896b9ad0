// Group norm with an activation, channels last, backward:
//   xh = (x - mean) rstd,  dz = dy f'(gamma xh + beta),  dgamma = sum dz xh,  dbeta = sum dz,
//   dx = rstd (gamma dz - m1 - xh m2),  m1, m2 = means over the group of gamma dz and gamma dz xh,
// which are sums over the group's channels of gamma times the channel's two sums.
// Any shape in three steps: both sums per channel of a chunk of pixels; joined per group and over the samples; the elements.
//   32 x 3136 x 256 bf16, SiLU, x kept: 32 us, 4 and 31.  Both large steps compute the slope, 20 instructions an element of which two go to the
// exponential pipe (40 % busy); without it they take 19 and 20 us, which is what their bytes take.
#include "ogq_group_norm_resident.cuh"

namespace ogq {

// What the backward pass reads of V channels of a pixel: dy, and x as it is or as it was kept.
template <class E, int V, bool KEPT>
struct GnPair {
    GnRaw<E, V> dy;
    std::conditional_t<KEPT, GnKept<V>, GnRaw<E, V>> x;
    // dz, and x less the mean
    template <int ACT, bool ACCURATE>
    __device__ __forceinline__ void open(int act, const GnAffine<V>& f, float (&dz)[V], float (&xc)[V]) const
    {
        gn_open<E, V>(dy, dz);
        if constexpr (KEPT) gn_open<V>(x, xc);
        else gn_open<E, V>(x, xc);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            xc[j] = f.centre(xc[j], j);
            dz[j] = __fmul_rn(dz[j], gn_slope<ACT, ACCURATE>(act, f.z(xc[j], j)));
        }
    }
};

// The pointers of a thread's first pixel and how far the next one's are.
template <class E, int V, bool KEPT>
struct GnReader {
    const E *dy, *x;
    const int8_t* codes;
    const uint8_t* scales;
    int step, scale_step;
    __device__ __forceinline__ GnReader(const GnArgs& a, const GnPlace& q)
    {
        const int groups = (int)act8_groups(a.t.C);
        const int64_t at = q.row * a.t.C + q.c;
        dy = (const E*)a.dy + at;
        x = KEPT ? nullptr : (const E*)a.x + at;
        codes = KEPT ? a.codes + at : nullptr;
        scales = KEPT ? a.scales + q.row * groups + (uint32_t)q.c / kAct8Group : nullptr;
        step = a.t.ty * (int)a.t.C;
        scale_step = a.t.ty * groups;
    }
    __device__ __forceinline__ void fetch(int i, GnPair<E, V, KEPT>& r) const
    {
        r.dy = gn_fetch<E, V>(dy + (int64_t)i * step);
        if constexpr (KEPT) r.x = gn_fetch_kept<V>(codes + (int64_t)i * step, scales + (int64_t)i * scale_step);
        else r.x = gn_fetch<E, V>(x + (int64_t)i * step);
    }
};

// Three CTAs an SM for 16-bit types (113.5 us a pass of the shape above, 115.8 with the two that 98 registers leave); fp32 spills at 80
// registers (4 x 16384 x 256, GELU: 128 us a pass against 116).
template <class E, int V, int ACT, bool KEPT>
__global__ void __launch_bounds__(kThreads, sizeof(E) == 4 ? 2 : 3) k_gn_grad_sums(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    __shared__ float2 sh[kThreads * V];
    const GnPlace q = gn_place<V>(a.t);
    if (q.active) {
        const GnReader<E, V, KEPT> in(a, q);
        GnAffine<V> f;  // sums of dz (x - mean): less the mean first, so that nothing is lost when they cancel
        gn_affine(a, q.n, q.c, f);
        float sb[V], sg[V];
#pragma unroll
        for (int j = 0; j < V; ++j) sb[j] = sg[j] = 0.f;
        gn_pixels<GnPair<E, V, KEPT>, 1>(q.count, [&](int i, GnPair<E, V, KEPT>& r) { in.fetch(i, r); },
                                      [&](int, const GnPair<E, V, KEPT>& r) {
                                          float dz[V], xc[V];
                                          r.template open<ACT, kAccurate>(a.act, f, dz, xc);
#pragma unroll
                                          for (int j = 0; j < V; ++j) {
                                              sb[j] = __fadd_rn(sb[j], dz[j]);
                                              sg[j] = __fmaf_rn(dz[j], xc[j], sg[j]);
                                          }
                                      });
        gn_channels<V>(a, q.n, q.c, [&](int j, float, float rstd, int64_t) {
            sh[(q.ty * a.t.tx + q.tx) * V + j] = make_float2(sb[j], __fmul_rn(sg[j], rstd));
        });
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.t.tx * V; j += kThreads) {
        const int64_t c = (int64_t)q.tile * a.t.tx * V + j;
        if (c >= a.t.C) break;
        double s1 = 0.0, s2 = 0.0;  // up to 256 rows, one after the other, of sums that may cancel
        for (int y = 0; y < a.t.ty; ++y) {
            const float2 e = sh[y * a.t.tx * V + j];
            s1 += (double)e.x;
            s2 += (double)e.y;
        }
        a.part[((int64_t)q.n * a.t.chunks + q.chunk) * a.t.C + c] = make_float2((float)s1, (float)s2);
    }
}

// The first CTAs: one per sample and group, m1 and m2.  The others: dgamma and dbeta of eight channels each, 32 rows of partial
// sums at a time.
__global__ void __launch_bounds__(kThreads) k_gn_grad_join(const __grid_constant__ GnArgs a, int group_ctas)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ double sh[2][kThreads];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if ((int)blockIdx.x < group_ctas) {
        const int64_t w = blockIdx.x;
        const int n = (int)(w / a.t.G), g = (int)(w - n * a.t.G), per = (int)(a.t.C / a.t.G);
        const int64_t entries = (int64_t)a.t.chunks * per;
        const float2* part = a.part + (int64_t)n * a.t.chunks * a.t.C + (int64_t)g * per;
        double s1 = 0.0, s2 = 0.0;
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < entries; i += kThreads) {
            const uint32_t k = (uint32_t)i / (uint32_t)per, c = (uint32_t)i - k * per;
            const float2 e = __ldcg(part + (int64_t)k * a.t.C + c);
            const double gamma = a.gamma ? (double)a.gamma[(int64_t)g * per + c] : 1.0;
            s1 += gamma * (double)e.x;
            s2 += gamma * (double)e.y;
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (lane == 0) {
            sh[0][warp] = s1;
            sh[1][warp] = s2;
        }
        __syncthreads();
        const double m = (double)(a.t.P * per);
        if (threadIdx.x == 0) {
            s1 = s2 = 0.0;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) {
                s1 += sh[0][i];
                s2 += sh[1][i];
            }
            a.sums[w] = make_float2((float)(s1 / m), (float)(s2 / m));
        }
        return;
    }
    const int64_t c = (int64_t)((int)blockIdx.x - group_ctas) * 8 + (threadIdx.x & 7);
    double sb = 0.0, sg = 0.0;
    if (c < a.t.C) {
#pragma unroll 4
        for (int64_t r = threadIdx.x >> 3; r < a.N * a.t.chunks; r += kThreads / 8) {
            const float2 e = __ldcg(a.part + r * a.t.C + c);
            sb += (double)e.x;
            sg += (double)e.y;
        }
    }
    sh[0][threadIdx.x] = sb;
    sh[1][threadIdx.x] = sg;
    __syncthreads();
    if (threadIdx.x < 16) {  // eight channels of both
        const int which = threadIdx.x >> 3;
        const int64_t o = (int64_t)((int)blockIdx.x - group_ctas) * 8 + (threadIdx.x & 7);
        double s = 0.0;
        for (int k = 0; k < kThreads / 8; ++k) s += sh[which][k * 8 + (threadIdx.x & 7)];
        float* out = which ? a.dgamma : a.dbeta;
        if (out && o < a.t.C) out[o] = (float)s;
    }
}

template <class E, int V, int ACT, bool KEPT>
__global__ void __launch_bounds__(kThreads) k_gn_grad(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    const GnPlace q = gn_place<V>(a.t);
    if (!q.active) return;
    const GnReader<E, V, KEPT> in(a, q);
    GnAffine<V> f;
    gn_affine(a, q.n, q.c, f);
    float slope[V], offset[V];
    gn_channels<V>(a, q.n, q.c, [&](int j, float, float rstd, int64_t at) {
        gn_gradient_terms(__ldcg(a.sums + at), rstd, slope[j], offset[j]);
    });
    E* out = (E*)a.out + q.row * a.t.C + q.c;
    gn_pixels<GnPair<E, V, KEPT>, sizeof(E) == 2 ? 2 : 1>(q.count, [&](int i, GnPair<E, V, KEPT>& r) { in.fetch(i, r); },
                                  [&](int i, const GnPair<E, V, KEPT>& r) {
                                      float dz[V], xc[V];
                                      r.template open<ACT, kAccurate>(a.act, f, dz, xc);
#pragma unroll
                                      for (int j = 0; j < V; ++j) dz[j] = __fmaf_rn(dz[j], f.scale[j], __fmaf_rn(xc[j], slope[j], offset[j]));
                                      gn_store(out + (int64_t)i * in.step, dz);
                                  });
}

// The whole pass of one slab (see ogq_group_norm_resident.cuh): dy and x are read once, dz stays in fp32 registers (its slope costs
// more than its 8 registers a vector), xh is computed again from x.
template <class E, int ACT, bool KEPT, int U>
__global__ void __launch_bounds__(kThreads, U <= 2 ? 3 : 2) k_gn_backward(const __grid_constant__ GnArgs a, const __grid_constant__ GnSlab s)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    __shared__ float2 sh[kThreads * 8];
    __shared__ float2 sh_cta[kGnMaxWidth], sh_all[kGnMaxWidth], sh_group[kGnMaxWidth];
    const GnSpot q = gn_spot(a.t, s);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int groups = s.width / s.per;
    Raw8<E> rdy[U], rx[KEPT ? 1 : U];
    uint2 kx[KEPT ? U : 1];
    uint32_t ks[KEPT ? U : 1];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t p = q.first + q.ty + u * s.rows;
        in[u] = q.active && p < q.last;
        const int64_t row = q.n * a.t.P + p;
        rdy[u] = in[u] ? load_raw8((const E*)a.dy + row * a.t.C + q.c) : zero_raw8<E>();
        if constexpr (KEPT) {
            kx[u] = make_uint2(0u, 0u);
            ks[u] = 0u;
            if (in[u]) {
                kx[u] = *reinterpret_cast<const uint2*>(a.codes + row * a.t.C + q.c);
                ks[u] = a.scales[row * act8_groups(a.t.C) + q.c / kAct8Group];
            }
        } else {
            rx[u] = in[u] ? load_raw8((const E*)a.x + row * a.t.C + q.c) : zero_raw8<E>();
        }
    }
    GnAffine<8> z;
    if (q.active) gn_affine(a, q.n, q.c, z);
    float dz[U][8];
    float2 sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = make_float2(0.f, 0.f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        unpack8(rdy[u], dz[u]);
        if constexpr (KEPT) act8_values(kx[u], act8_unit(ks[u]), f);
        else unpack8(rx[u], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float xc = z.centre(f[j], j);
            dz[u][j] = __fmul_rn(dz[u][j], act_slope<ACT, kAccurate>(z.z(xc, j)));
            if (in[u]) {
                sum[j].x = __fadd_rn(sum[j].x, dz[u][j]);
                sum[j].y = __fmaf_rn(dz[u][j], xc, sum[j].y);
            }
        }
    }
    if (q.active)
        gn_channels<8>(a, q.n, q.c, [&](int j, float, float rstd, int64_t) { sum[j].y = __fmul_rn(sum[j].y, rstd); });
    gn_put_sums(s, q, sum, sh, s.width);
    __syncthreads();
    for (int c = threadIdx.x; c < s.width; c += kThreads) {
        float2 t = make_float2(0.f, 0.f);
        for (int r = 0; r < s.sum_rows; ++r) {
            const float2 e = sh[r * s.width + c];
            t.x += e.x;
            t.y += e.y;
        }
        sh_cta[c] = t;
    }
    if (s.cluster > 1) {
        gn_cluster_arrive();
        gn_cluster_wait();
    } else {
        __syncthreads();
    }
    for (int c = threadIdx.x; c < s.width; c += kThreads) {
        float2 t = sh_cta[c];
        if (s.cluster > 1) {
            t = make_float2(0.f, 0.f);
            float2 e[kGnMaxCluster];  // all under way before the first is added
#pragma unroll
            for (int r = 0; r < kGnMaxCluster; ++r) e[r] = r < s.cluster ? gn_remote(&sh_cta[c], r) : make_float2(0.f, 0.f);
#pragma unroll
            for (int r = 0; r < kGnMaxCluster; ++r) {
                t.x += e[r].x;
                t.y += e[r].y;
            }
        }
        const int64_t at = q.c - q.c0 + c;
        if (q.rank == 0) {
            if (a.N > 1) {
                a.part[q.n * a.t.C + at] = t;
            } else {  // nothing to add up
                if (a.dbeta) a.dbeta[at] = t.x;
                if (a.dgamma) a.dgamma[at] = t.y;
            }
        }
        const float gamma = a.gamma ? a.gamma[at] : 1.f;
        sh_all[c] = make_float2(gamma * t.x, gamma * t.y);
    }
    __syncthreads();
    if (s.cluster > 1) gn_cluster_arrive();  // this CTA has read the others' sums
    for (int g = warp; g < groups; g += kWarps) {
        float2 t = make_float2(0.f, 0.f);
        for (int c = lane; c < s.per; c += 32) {
            t.x += sh_all[g * s.per + c].x;
            t.y += sh_all[g * s.per + c].y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
            t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
        }
        const float m = (float)(a.t.P * s.per);
        if (lane == 0) sh_group[g] = make_float2(t.x / m, t.y / m);
    }
    __syncthreads();
    if (q.active) {
        float slope[8], offset[8];
        const int64_t base = q.n * a.t.G + (int)(q.c - q.c0) / s.per;  // the slab's first group
        gn_channels<8>(a, q.n, q.c, [&](int j, float, float rstd, int64_t at) {
            gn_gradient_terms(sh_group[at - base], rstd, slope[j], offset[j]);
        });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            const int64_t row = q.n * a.t.P + q.first + q.ty + u * s.rows;
            float f[8];
            if constexpr (KEPT) act8_values(kx[u], act8_unit(ks[u]), f);
            else unpack8(rx[u], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __fmaf_rn(dz[u][j], z.scale[j], __fmaf_rn(z.centre(f[j], j), slope[j], offset[j]));
            store8((E*)a.out + row * a.t.C + q.c, f);
        }
    }
    if (s.cluster > 1) gn_cluster_wait();  // the others have read this CTA's
}

cudaError_t launch_group_norm_backward(const GroupNorm& p, int sm_count, cudaStream_t stream)
{
    const size_t size = p.dtype == OGQ_F32 ? 4 : 2;
    const bool kept = p.codes != nullptr;
    const bool vec = p.C % 8 == 0 && gn_aligned(p.dy, 16) && gn_aligned(p.out, 16) && (p.C * size) % 16 == 0 &&
                     (kept ? gn_aligned(p.codes, 8) : gn_aligned(p.x, 16));
    GnArgs a = gn_args(p, gn_tiles(p.N, p.P, p.C, p.G, vec ? 8 : 1, sm_count, 1));
    const int channel_ctas = p.dgamma || p.dbeta ? (int)((p.C + 7) / 8) : 0;
    GnSlab slab;
    if (vec && a.t.ctas > 0) {
        const int u = gn_vectors(p.N, p.P, p.C, p.G, (int)size, false, 4, kGnBackwardWork, sm_count, slab);
        if (u) {
            launch_begin("k_gn_backward", stream);
            cudaError_t e = with_dtype(p.dtype, [&](auto elem) {
                using E = decltype(elem);
                return with_act(p.act, [&](auto act) {
                    constexpr int A = decltype(act)::value;
                    return with_bool(kept, [&](auto k) {
                        constexpr bool K = decltype(k)::value;
                        return u == 2 ? launch_cluster(k_gn_backward<E, A, K, 2>, slab.ctas, slab.cluster, stream, a, slab)
                                      : launch_cluster(k_gn_backward<E, A, K, 4>, slab.ctas, slab.cluster, stream, a, slab);
                    });
                });
            });
            launch_end(stream);
            if (e != cudaSuccess || channel_ctas == 0 || p.N == 1) return e;
            a.t.chunks = 1;  // a pair of sums per sample and channel
            launch_begin("k_gn_grad_join", stream);
            e = launch_pdl(k_gn_grad_join, channel_ctas, kThreads, 0, stream, a, 0);
            launch_end(stream);
            return e;
        }
    }
    if (a.t.ctas > 0x7fffffff) return cudaErrorInvalidValue;
    const auto launch = [&](auto which) {
        constexpr bool kSums = decltype(which)::value;
        const auto one = [&](auto kernel, int V) {
            a = gn_args(p, gn_tiles(p.N, p.P, p.C, p.G, V, gn_wave(kernel, sm_count), kSums ? kGnMinChunk : 2));
            if (a.t.ctas == 0) return cudaSuccess;
            launch_begin(kSums ? "k_gn_grad_sums" : "k_gn_grad", stream);
            const cudaError_t r = launch_pdl(kernel, (int)a.t.ctas, kThreads, 0, stream, a);
            launch_end(stream);
            return r;
        };
        return with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            return with_bool(kept, [&](auto k) {
                constexpr bool K = decltype(k)::value;
                if (!vec) return one(kSums ? k_gn_grad_sums<E, 1, -1, K> : k_gn_grad<E, 1, -1, K>, 1);
                return with_act(p.act, [&](auto act) {
                    constexpr int A = decltype(act)::value;
                    return one(kSums ? k_gn_grad_sums<E, 8, A, K> : k_gn_grad<E, 8, A, K>, 8);
                });
            });
        });
    };
    const bool any = a.t.ctas > 0;
    cudaError_t e = launch(std::true_type{});
    if (e != cudaSuccess) return e;
    const int group_ctas = any ? (int)(p.N * p.G) : 0;
    const auto join = [&](int groups, int channels) {
        if (groups + channels == 0) return cudaSuccess;
        launch_begin("k_gn_grad_join", stream);
        const cudaError_t r = launch_pdl(k_gn_grad_join, groups + channels, kThreads, 0, stream, a, groups);
        launch_end(stream);
        return r;
    };
    if ((int64_t)group_ctas + channel_ctas <= 0x7fffffff) {
        e = join(group_ctas, channel_ctas);
    } else {  // more than a grid holds
        e = join(group_ctas, 0);
        if (e == cudaSuccess) e = join(0, channel_ctas);
    }
    if (e != cudaSuccess || !any) return e;
    return launch(std::false_type{});
}

}  // namespace ogq

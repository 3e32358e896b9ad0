// Group norm with an activation, channels last, backward:
//   xh = (x - mean) rstd,  dz = dy f'(gamma xh + beta),  dgamma = sum dz xh,  dbeta = sum dz,
//   dx = rstd (gamma dz - m1 - xh m2),  m1, m2 = means over the group of gamma dz and gamma dz xh,
// which are sums over the group's channels of gamma times the channel's two sums.
// Any shape in three steps: both sums per channel of a chunk of pixels; joined per group and over the samples; the elements.
#include "ogq_group_norm.cuh"

namespace ogq {

// dz and xh of V channels of a pixel
template <class E, int V, int ACT, bool KEPT>
__device__ __forceinline__ void gn_dz(const GnArgs& a, int64_t row, int64_t c, const GnChannels<V>& ch, float (&dz)[V], float (&xh)[V])
{
    constexpr bool kAccurate = sizeof(E) == 4;
    gn_load((const E*)a.dy + row * a.t.C + c, dz);
    if constexpr (KEPT) gn_kept(a.codes, a.scales, row, a.t.C, c, xh);
    else gn_load((const E*)a.x + row * a.t.C + c, xh);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        xh[j] = __fmul_rn(__fsub_rn(xh[j], ch.mean[j]), ch.rstd[j]);
        dz[j] = __fmul_rn(dz[j], gn_slope<ACT, kAccurate>(a.act, __fmaf_rn(xh[j], ch.gamma[j], ch.beta[j])));
    }
}

template <class E, int V, int ACT, bool KEPT>
__global__ void __launch_bounds__(kThreads) k_gn_grad_sums(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float2 sh[kThreads * V];
    const GnPlace q = gn_place<V>(a.t);
    if (q.active) {
        GnChannels<V> ch;
        ch.load(a, q.n, q.c);
        float sb[V], sg[V];
#pragma unroll
        for (int j = 0; j < V; ++j) sb[j] = sg[j] = 0.f;
        for (int64_t p = q.first; p < q.last; p += a.t.ty) {
            float dz[V], xh[V];
            gn_dz<E, V, ACT, KEPT>(a, q.n * a.t.P + p, q.c, ch, dz, xh);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sb[j] = __fadd_rn(sb[j], dz[j]);
                sg[j] = __fmaf_rn(dz[j], xh[j], sg[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sh[(q.ty * a.t.tx + q.tx) * V + j] = make_float2(sb[j], sg[j]);
    }
    __syncthreads();
    const int tile = (int)(blockIdx.x % (unsigned)a.t.ctiles);
    for (int j = threadIdx.x; j < a.t.tx * V; j += kThreads) {
        const int64_t c = (int64_t)tile * a.t.tx * V + j;
        if (c >= a.t.C) break;
        float2 s = make_float2(0.f, 0.f);
        for (int y = 0; y < a.t.ty; ++y) {
            const float2 e = sh[y * a.t.tx * V + j];
            s.x += e.x;
            s.y += e.y;
        }
        a.part[(q.n * a.t.chunks + q.chunk) * a.t.C + c] = s;
    }
}

// The first CTAs: a warp per sample and group, m1 and m2.  The others: dgamma and dbeta of 32 channels each.
__global__ void __launch_bounds__(kThreads) k_gn_grad_join(const __grid_constant__ GnArgs a, int group_ctas)
{
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if ((int)blockIdx.x < group_ctas) {
        const int64_t w = (int64_t)blockIdx.x * kWarps + warp;
        if (w >= a.N * a.t.G) return;
        const int64_t n = w / a.t.G, g = w - n * a.t.G, per = a.t.C / a.t.G;
        const int64_t entries = a.t.chunks * per;
        const float2* part = a.part + n * a.t.chunks * a.t.C + g * per;
        double s1 = 0.0, s2 = 0.0;
        for (int64_t i = lane; i < entries; i += 32) {
            const int64_t k = i / per, c = i - k * per;
            const float2 e = __ldcg(part + k * a.t.C + c);
            const double gamma = a.gamma ? (double)a.gamma[g * per + c] : 1.0;
            s1 += gamma * (double)e.x;
            s2 += gamma * (double)e.y;
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        const double m = (double)(a.t.P * per);
        if (lane == 0) a.sums[w] = make_float2((float)(s1 / m), (float)(s2 / m));
        return;
    }
    __shared__ double sh[2][kWarps][32];
    const int64_t c = (int64_t)((int)blockIdx.x - group_ctas) * 32 + lane;
    double sb = 0.0, sg = 0.0;
    if (c < a.t.C) {
        for (int64_t r = warp; r < a.N * a.t.chunks; r += kWarps) {
            const float2 e = __ldcg(a.part + r * a.t.C + c);
            sb += (double)e.x;
            sg += (double)e.y;
        }
    }
    sh[0][warp][lane] = sb;
    sh[1][warp][lane] = sg;
    __syncthreads();
    if (warp < 2 && c < a.t.C) {
        double s = 0.0;
        for (int k = 0; k < kWarps; ++k) s += sh[warp][k][lane];
        float* out = warp ? a.dgamma : a.dbeta;
        if (out) out[c] = (float)s;
    }
}

template <class E, int V, int ACT, bool KEPT>
__global__ void __launch_bounds__(kThreads) k_gn_grad(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    const GnPlace q = gn_place<V>(a.t);
    if (!q.active) return;
    GnChannels<V> ch;
    ch.load(a, q.n, q.c);
    float m1[V], m2[V];
    const int64_t per = a.t.C / a.t.G;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 s = __ldcg(a.sums + q.n * a.t.G + (q.c + j) / per);
        m1[j] = s.x;
        m2[j] = s.y;
    }
    for (int64_t p = q.first; p < q.last; p += a.t.ty) {
        const int64_t row = q.n * a.t.P + p;
        float dz[V], xh[V], dx[V];
        gn_dz<E, V, ACT, KEPT>(a, row, q.c, ch, dz, xh);
#pragma unroll
        for (int j = 0; j < V; ++j)
            dx[j] = __fmul_rn(ch.rstd[j], __fmaf_rn(-xh[j], m2[j], __fmaf_rn(dz[j], ch.gamma[j], -m1[j])));
        gn_store((E*)a.out + row * a.t.C + q.c, dx);
    }
}

cudaError_t launch_group_norm_backward(const GroupNorm& p, int sm_count, cudaStream_t stream)
{
    const size_t size = p.dtype == OGQ_F32 ? 4 : 2;
    const bool kept = p.codes != nullptr;
    const bool vec = p.C % 8 == 0 && gn_aligned(p.dy, 16) && gn_aligned(p.out, 16) && (p.C * size) % 16 == 0 &&
                     (kept ? gn_aligned(p.codes, 8) : gn_aligned(p.x, 16));
    const GnArgs a = gn_args(p, gn_tiles(p.N, p.P, p.C, p.G, vec ? 8 : 1, sm_count));
    const auto launch = [&](auto which) {
        constexpr bool kSums = decltype(which)::value;
        return with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            return with_bool(kept, [&](auto k) {
                constexpr bool K = decltype(k)::value;
                if (!vec) return launch_pdl(kSums ? k_gn_grad_sums<E, 1, -1, K> : k_gn_grad<E, 1, -1, K>, (int)a.t.ctas, kThreads, 0, stream, a);
                return with_act(p.act, [&](auto act) {
                    constexpr int A = decltype(act)::value;
                    return launch_pdl(kSums ? k_gn_grad_sums<E, 8, A, K> : k_gn_grad<E, 8, A, K>, (int)a.t.ctas, kThreads, 0, stream, a);
                });
            });
        });
    };
    cudaError_t e = cudaSuccess;
    if (a.t.ctas > 0) {
        launch_begin("k_gn_grad_sums", stream);
        e = launch(std::true_type{});
        launch_end(stream);
        if (e != cudaSuccess) return e;
    }
    const int group_ctas = a.t.ctas > 0 ? (int)((p.N * p.G + kWarps - 1) / kWarps) : 0;
    const int channel_ctas = p.dgamma || p.dbeta ? (int)((p.C + 31) / 32) : 0;
    if (group_ctas + channel_ctas > 0) {
        launch_begin("k_gn_grad_join", stream);
        e = launch_pdl(k_gn_grad_join, group_ctas + channel_ctas, kThreads, 0, stream, a, group_ctas);
        launch_end(stream);
    }
    if (e != cudaSuccess || a.t.ctas == 0) return e;
    launch_begin("k_gn_grad", stream);
    e = launch(std::false_type{});
    launch_end(stream);
    return e;
}

}  // namespace ogq

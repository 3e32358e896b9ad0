// Group norm with an activation, channels last, forward:
//   mean, rstd over the P x C/G values of a group of a sample;  y = f(gamma (x - mean) rstd + beta)
// Any shape in three steps: moments per channel of a chunk of pixels, joined per group, then the elements.
//   Moments are sums about the first value a thread sees: that value is one of those summed, so the sum of squares about the
// mean is at least (1 - 1/n) of its squared distance d to the mean, while what is subtracted is n d^2: with n <= 64 pixels a thread the
// difference loses at most a factor 64 of fp32's 2^-24.  Joining two sets adds n_a n_b / (n_a + n_b) (mean_a - mean_b)^2, all positive.
#include "ogq_group_norm.cuh"

namespace ogq {

template <class E, int V>
__global__ void __launch_bounds__(kThreads) k_gn_moments(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float2 sh[kThreads * V];
    const GnPlace q = gn_place<V>(a.t);
    float shift[V], s1[V], s2[V];
    int n = 0;
    if (q.active) {
        const E* x = (const E*)a.x + q.n * a.t.P * a.t.C + q.c;
#pragma unroll
        for (int j = 0; j < V; ++j) s1[j] = s2[j] = shift[j] = 0.f;
        for (int64_t p = q.first; p < q.last; p += a.t.ty, ++n) {
            float v[V];
            gn_load(x + p * a.t.C, v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (n == 0) shift[j] = v[j];
                const float d = __fsub_rn(v[j], shift[j]);
                s1[j] = __fadd_rn(s1[j], d);
                s2[j] = __fmaf_rn(d, d, s2[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float m = n ? s1[j] / (float)n : 0.f;
            sh[(q.ty * a.t.tx + q.tx) * V + j] = make_float2(shift[j] + m, fmaxf(__fmaf_rn(-m, s1[j], s2[j]), 0.f));
        }
    }
    __syncthreads();
    // pixels of the rows of threads: row y has `whole` and, if y < more, one more
    const int64_t begin = (int64_t)q.chunk * a.t.ty * a.t.px;
    const int count = (int)(q.last - begin), whole = count / a.t.ty, more = count - whole * a.t.ty;
    const int tile = (int)(blockIdx.x % (unsigned)a.t.ctiles);
    for (int j = threadIdx.x; j < a.t.tx * V; j += kThreads) {
        const int64_t c = (int64_t)tile * a.t.tx * V + j;
        if (c >= a.t.C) break;
        float sum = 0.f;
        for (int y = 0; y < a.t.ty; ++y) sum += (float)(whole + (y < more)) * sh[y * a.t.tx * V + j].x;
        const float mean = sum / (float)count;
        float m2 = 0.f;
        for (int y = 0; y < a.t.ty; ++y) {
            const float2 e = sh[y * a.t.tx * V + j];
            const float d = e.x - mean, w = (float)(whole + (y < more));
            m2 += w > 0.f ? __fmaf_rn(w * d, d, e.y) : 0.f;
        }
        a.part[(q.n * a.t.chunks + q.chunk) * a.t.C + c] = make_float2(mean, m2);
    }
}

// A warp per sample and group: joins the channels and chunks.
__global__ void __launch_bounds__(kThreads) k_gn_stats(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (w >= a.N * a.t.G) return;
    const int64_t n = w / a.t.G, g = w - n * a.t.G, per = a.t.C / a.t.G;
    const int64_t px = (int64_t)a.t.ty * a.t.px;
    const int64_t entries = a.t.chunks * per;
    const float2* part = a.part + n * a.t.chunks * a.t.C + g * per;
    double sum = 0.0;
    for (int64_t i = lane; i < entries; i += 32) {
        const int64_t k = i / per, c = i - k * per;
        const int64_t count = (k + 1) * px < a.t.P ? px : a.t.P - k * px;
        sum += (double)count * (double)__ldcg(part + k * a.t.C + c).x;
    }
    const double m = (double)(a.t.P * per);
    const double mean = m > 0 ? warp_sum(sum) / m : 0.0;
    double m2 = 0.0;
    for (int64_t i = lane; i < entries; i += 32) {
        const int64_t k = i / per, c = i - k * per;
        const int64_t count = (k + 1) * px < a.t.P ? px : a.t.P - k * px;
        const float2 e = __ldcg(part + k * a.t.C + c);
        const double d = (double)e.x - mean;
        m2 += (double)e.y + (double)count * d * d;
    }
    m2 = warp_sum(m2);
    if (lane == 0) {
        a.mean[w] = (float)mean;
        a.rstd[w] = (float)(1.0 / sqrt((m > 0 ? m2 / m : 0.0) + (double)a.eps));
    }
}

// KEEP: 0 nothing, 1 codes to nearest, 2 codes at random (V = 8 and whole groups of 32 channels: four lanes hold a group)
template <class E, int V, int ACT, int KEEP>
__global__ void __launch_bounds__(kThreads) k_gn_apply(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    const GnPlace q = gn_place<V>(a.t);
    if (!q.active) return;  // KEEP: whole groups of lanes, since tx is a multiple of 4
    GnChannels<V> ch;
    ch.load(a, q.n, q.c);
    float scale[V];
#pragma unroll
    for (int j = 0; j < V; ++j) scale[j] = ch.rstd[j] * ch.gamma[j];
    const unsigned team = 0xfu << (threadIdx.x & 28);
    for (int64_t p = q.first; p < q.last; p += a.t.ty) {
        const int64_t row = q.n * a.t.P + p;
        float v[V], y[V];
        gn_load((const E*)a.x + row * a.t.C + q.c, v);
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = gn_value<ACT, kAccurate>(a.act, __fmaf_rn(__fsub_rn(v[j], ch.mean[j]), scale[j], ch.beta[j]));
        if constexpr (KEEP != 0 && V == 8) {
            const uint32_t byte = act8_byte(__reduce_max_sync(team, max_abs_bits(v)));
            *reinterpret_cast<uint2*>(a.codes + row * a.t.C + q.c) =
                act8_codes<KEEP == 2>(v, byte, (uint64_t)(row * a.t.C + q.c), 0u, a.stream_id, a.keys);
            if ((threadIdx.x & 3) == 0) a.scales[(row * a.t.C + q.c) / kAct8Group] = (uint8_t)byte;
        }
        gn_store((E*)a.out + row * a.t.C + q.c, y);
    }
}

size_t ws_bytes_group_norm(int64_t N, int64_t P, int64_t C, int64_t G)
{
    if (N == 0 || C == 0) return 0;
    return gn_part_bytes(N, P, C) + ((size_t)(N * G) * sizeof(float2) + 255) / 256 * 256;
}

cudaError_t launch_group_norm_forward(const GroupNorm& p, int sm_count, cudaStream_t stream)
{
    const size_t size = p.dtype == OGQ_F32 ? 4 : 2;
    const bool vec = p.C % 8 == 0 && gn_aligned(p.x, 16) && gn_aligned(p.out, 16) && (p.C * size) % 16 == 0;
    const bool fused = p.codes && vec && p.C % kAct8Group == 0 && gn_aligned(p.codes, 8);
    cudaError_t e = cudaSuccess;
    if (p.codes && !fused && p.P > 0) {  // before the elements: y may be x
        Act8Forward f = {};
        f.x = p.x; f.ld_x = p.C; f.rows = p.N * p.P; f.cols = p.C;
        f.dtype = p.dtype; f.rounding = p.rounding; f.seed = p.seed; f.stream_id = p.stream_id;
        f.codes = p.codes; f.scales = p.scales;
        e = launch_act8_forward(f, sm_count, stream);
        if (e != cudaSuccess) return e;
    }
    const GnArgs a = gn_args(p, gn_tiles(p.N, p.P, p.C, p.G, vec ? 8 : 1, sm_count));
    if (a.t.ctas > 0) {
        launch_begin("k_gn_moments", stream);
        e = with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            return vec ? launch_pdl(k_gn_moments<E, 8>, (int)a.t.ctas, kThreads, 0, stream, a)
                       : launch_pdl(k_gn_moments<E, 1>, (int)a.t.ctas, kThreads, 0, stream, a);
        });
        launch_end(stream);
        if (e != cudaSuccess) return e;
    }
    launch_begin("k_gn_stats", stream);
    e = launch_pdl(k_gn_stats, (int)((p.N * p.G + kWarps - 1) / kWarps), kThreads, 0, stream, a);
    launch_end(stream);
    if (e != cudaSuccess || a.t.ctas == 0) return e;
    launch_begin("k_gn_apply", stream);
    e = with_dtype(p.dtype, [&](auto elem) {
        using E = decltype(elem);
        if (!vec) return launch_pdl(k_gn_apply<E, 1, -1, 0>, (int)a.t.ctas, kThreads, 0, stream, a);
        return with_act(p.act, [&](auto act) {
            constexpr int A = decltype(act)::value;
            if (!fused) return launch_pdl(k_gn_apply<E, 8, A, 0>, (int)a.t.ctas, kThreads, 0, stream, a);
            if (p.rounding == OGQ_ROUND_RANDOM) return launch_pdl(k_gn_apply<E, 8, A, 2>, (int)a.t.ctas, kThreads, 0, stream, a);
            return launch_pdl(k_gn_apply<E, 8, A, 1>, (int)a.t.ctas, kThreads, 0, stream, a);
        });
    });
    launch_end(stream);
    return e;
}

}  // namespace ogq

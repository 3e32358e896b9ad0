// Group norm with an activation, channels last, forward:
//   mean, rstd over the P x C/G values of a group of a sample;  y = f(gamma (x - mean) rstd + beta)
// Any shape in three steps: moments per channel of a chunk of pixels, joined per group, then the elements.
//   32 x 3136 x 256 bf16, SiLU, x kept: 15 us of moments (51 MB, 3.4 TB/s: a load, a dozen instructions, the next), 5 of joining, 25 of elements
// (x from L2; 128 MB moved, the exponential pipe busy half the time).
//   Moments are sums about the first value a thread sees: that value is one of those summed, so the sum of squares about the
// mean is at least (1 - 1/n) of its squared distance d to the mean, while what is subtracted is n d^2: with n <= 64 pixels a thread the
// difference loses at most a factor 64 of fp32's 2^-24.  Joining two sets adds n_a n_b / (n_a + n_b) (mean_a - mean_b)^2, all positive.
#include "ogq_group_norm_resident.cuh"

namespace ogq {

template <class E, int V>
__global__ void __launch_bounds__(kThreads) k_gn_moments(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float2 sh[kThreads * V];
    const GnPlace q = gn_place<V>(a.t);
    if (q.active) {
        const E* x = (const E*)a.x + q.row * a.t.C + q.c;
        const int step = a.t.ty * (int)a.t.C;
        float shift[V], s1[V], s2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) s1[j] = s2[j] = shift[j] = 0.f;
        gn_pixels<GnRaw<E, V>, 2>(q.count, [&](int i, GnRaw<E, V>& r) { r = gn_fetch<E, V>(x + (int64_t)i * step); },
                               [&](int i, const GnRaw<E, V>& r) {
                                   float v[V];
                                   gn_open<E, V>(r, v);
                                   if (i == 0) {
#pragma unroll
                                       for (int j = 0; j < V; ++j) shift[j] = fabsf(v[j]) < INFINITY ? v[j] : 0.f;
                                   }
#pragma unroll
                                   for (int j = 0; j < V; ++j) {
                                       const float d = __fsub_rn(v[j], shift[j]);
                                       s1[j] = __fadd_rn(s1[j], d);
                                       s2[j] = __fmaf_rn(d, d, s2[j]);
                                   }
                               });
        const float inv = q.count > 0 ? 1.f / (float)q.count : 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float m = __fmul_rn(s1[j], inv);
            sh[(q.ty * a.t.tx + q.tx) * V + j] = make_float2(shift[j] + m, fmaxf(__fmaf_rn(-m, s1[j], s2[j]), 0.f));
        }
    }
    __syncthreads();
    // pixels of the rows of threads: row y has `whole` and, if y < more, one more
    const int64_t begin = (int64_t)q.chunk * a.t.ty * a.t.px;
    const int count = (int)(a.t.P - begin < (int64_t)a.t.ty * a.t.px ? a.t.P - begin : (int64_t)a.t.ty * a.t.px);
    const int whole = (int)((uint32_t)count / (uint32_t)a.t.ty), more = count - whole * a.t.ty;
    const float inv = 1.f / (float)count, w0 = (float)whole, w1 = (float)(whole + 1);
    for (int j = threadIdx.x; j < a.t.tx * V; j += kThreads) {
        const int64_t c = (int64_t)q.tile * a.t.tx * V + j;
        if (c >= a.t.C) break;
        // about the first row's mean, which a chunk always has: the mean of one value everywhere is that value
        const float first = sh[j].x;
        float sum = 0.f;
        for (int y = 1; y < a.t.ty; ++y) sum = __fmaf_rn(y < more ? w1 : w0, whole || y < more ? __fsub_rn(sh[y * a.t.tx * V + j].x, first) : 0.f, sum);
        float mean = __fmaf_rn(sum, inv, first);
        if (mean != mean) {  // infinities: of one sign, the mean is theirs
            sum = 0.f;
            for (int y = 0; y < a.t.ty; ++y) sum = __fmaf_rn(y < more ? w1 : w0, whole || y < more ? sh[y * a.t.tx * V + j].x : 0.f, sum);
            mean = __fmul_rn(sum, inv);
        }
        float m2 = 0.f;
        for (int y = 0; y < a.t.ty; ++y) {
            const float2 e = sh[y * a.t.tx * V + j];
            const float d = e.x - mean;
            if (whole || y < more) m2 += __fmaf_rn((y < more ? w1 : w0) * d, d, e.y);
        }
        a.part[((int64_t)q.n * a.t.chunks + q.chunk) * a.t.C + c] = make_float2(mean, m2);
    }
}

// A CTA per sample and group: joins the channels and chunks.
__global__ void __launch_bounds__(kThreads) k_gn_stats(const __grid_constant__ GnArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ double scratch[2][kWarps];
    const int64_t w = blockIdx.x;
    const int n = (int)(w / a.t.G), g = (int)(w - n * a.t.G), per = (int)(a.t.C / a.t.G);
    const int64_t px = (int64_t)a.t.ty * a.t.px;
    const int64_t entries = (int64_t)a.t.chunks * per;  // below 2^31: no more than P C / G
    const float2* part = a.part + (int64_t)n * a.t.chunks * a.t.C + (int64_t)g * per;
    const auto entry = [&](int64_t i, double& count) {
        const uint32_t k = (uint32_t)i / (uint32_t)per, c = (uint32_t)i - k * per;
        count = (double)((k + 1) * px < a.t.P ? px : a.t.P - k * px);
        return __ldcg(part + (int64_t)k * a.t.C + c);
    };
    constexpr int kKeep = 4;  // entries a thread keeps between the two sums
    float2 kept[kKeep];
    double counts[kKeep];
    double sum = 0.0;
#pragma unroll
    for (int u = 0; u < kKeep; ++u) {
        counts[u] = 0.0;
        kept[u] = make_float2(0.f, 0.f);
        if (threadIdx.x + u * kThreads < entries) kept[u] = entry(threadIdx.x + u * kThreads, counts[u]);
    }
#pragma unroll
    for (int u = 0; u < kKeep; ++u)
        if (counts[u] > 0.0) sum += counts[u] * (double)kept[u].x;
    for (int64_t i = threadIdx.x + kKeep * kThreads; i < entries; i += kThreads) {
        double count;
        const float2 e = entry(i, count);
        sum += count * (double)e.x;
    }
    const double m = (double)(a.t.P * per);
    const auto total = [&](double v, double* sh) {
        v = warp_sum(v);
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
        __syncthreads();
        double t = 0.0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) t += sh[i];
        return t;
    };
    const double mean = m > 0 ? total(sum, scratch[0]) / m : 0.0;
    double m2 = 0.0;
#pragma unroll
    for (int u = 0; u < kKeep; ++u) {
        const double d = (double)kept[u].x - mean;
        if (counts[u] > 0.0) m2 += (double)kept[u].y + counts[u] * d * d;
    }
    for (int64_t i = threadIdx.x + kKeep * kThreads; i < entries; i += kThreads) {
        double count;
        const float2 e = entry(i, count);
        const double d = (double)e.x - mean;
        m2 += (double)e.y + count * d * d;
    }
    m2 = total(m2, scratch[1]);
    if (threadIdx.x == 0) {
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
    GnAffine<V> f;
    gn_affine(a, q.n, q.c, f);
    const unsigned team = 0xfu << (threadIdx.x & 28);
    const int64_t at = q.row * a.t.C + q.c;
    const int step = a.t.ty * (int)a.t.C;
    const E* x = (const E*)a.x + at;
    E* out = (E*)a.out + at;
    gn_pixels<GnRaw<E, V>, 2>(q.count, [&](int i, GnRaw<E, V>& r) { r = gn_fetch<E, V>(x + (int64_t)i * step); },
                           [&](int i, const GnRaw<E, V>& r) {
                               float v[V], y[V];
                               gn_open<E, V>(r, v);
                               const int64_t by = (int64_t)i * step;
                               if constexpr (KEEP != 0 && V == 8) {
                                   uint32_t b = max_abs_bits(r.e);
                                   b = max(b, __shfl_xor_sync(team, b, 1));
                                   b = max(b, __shfl_xor_sync(team, b, 2));
                                   const uint32_t byte = act8_byte(b);
                                   *reinterpret_cast<uint2*>(a.codes + at + by) =
                                       act8_codes<KEEP == 2>(v, byte, (uint64_t)(at + by), 0u, a.stream_id, a.keys);
                                   if ((threadIdx.x & 3) == 0) a.scales[(uint64_t)(at + by) / kAct8Group] = (uint8_t)byte;
                               }
#pragma unroll
                               for (int j = 0; j < V; ++j) y[j] = gn_value<ACT, kAccurate>(a.act, f.z(f.centre(v[j], j), j));
                               gn_store(out + by, y);
                           });
}

// The whole pass of one slab (see ogq_group_norm_resident.cuh): x is read once.  The CTA's mean, of plain sums; the sum of what deviates from it, which
// corrects it, and of the squares; then joined over the cluster about the first CTA's mean.  (Plain sums of one value c need not give c: 0.04 off after rstd = 316 at 1000.)
template <class E, int ACT, int KEEP, int U>
__global__ void __launch_bounds__(kThreads, U <= 2 ? 4 : U <= 4 ? 3 : 2) k_gn_forward(const __grid_constant__ GnArgs a, const __grid_constant__ GnSlab s)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    __shared__ float2 sh2[kThreads * 8];
    float* sh = reinterpret_cast<float*>(sh2);
    __shared__ float sh_mean[kGnMaxWidth], sh_rstd[kGnMaxWidth];
    __shared__ float2 sh_cta[kGnMaxWidth];
    const GnSpot q = gn_spot(a.t, s);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int groups = s.width / s.per;
    const E* x = (const E*)a.x + q.n * a.t.P * a.t.C + q.c;
    Raw8<E> v[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t p = q.first + q.ty + u * s.rows;
        in[u] = q.active && p < q.last;
        v[u] = in[u] ? load_raw8(x + p * a.t.C) : zero_raw8<E>();
    }
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        unpack8(v[u], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = __fadd_rn(sum[j], f[j]);  // pixels that are not there count 0
    }
    gn_put_sums(s, q, sum, sh, s.width);
    __syncthreads();
    const float count = (float)((int)(q.last - q.first) * s.per);
    for (int g = warp; g < groups; g += kWarps) {
        float t = 0.f;
        for (int c = lane; c < s.per; c += 32)
            for (int r = 0; r < s.sum_rows; ++r) t += sh[r * s.width + g * s.per + c];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        if (lane == 0) sh_mean[g] = count > 0.f ? t / count : 0.f;
    }
    __syncthreads();
    float m[8];
    float2 dev[8];
    {
        int g = q.c0 / s.per, left = (g + 1) * s.per - q.c0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (left == 0) { ++g; left = s.per; }
            --left;
            m[j] = sh_mean[g];
            dev[j] = make_float2(0.f, 0.f);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        unpack8(v[u], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = in[u] ? __fsub_rn(f[j], m[j]) : 0.f;
            dev[j].x = __fadd_rn(dev[j].x, d);
            dev[j].y = __fmaf_rn(d, d, dev[j].y);
        }
    }
    gn_put_sums(s, q, dev, sh2, s.width);
    __syncthreads();
    for (int g = warp; g < groups; g += kWarps) {
        float2 t = make_float2(0.f, 0.f);
        for (int c = lane; c < s.per; c += 32)
            for (int r = 0; r < s.sum_rows; ++r) {
                const float2 e = sh2[r * s.width + g * s.per + c];
                t.x += e.x;
                t.y += e.y;
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
            t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
        }
        const float by = count > 0.f ? t.x / count : 0.f;
        if (lane == 0) {
            const float m2 = __fmaf_rn(-by, t.x, t.y);
            const float m = sh_mean[g];
            sh_cta[g] = make_float2(fabsf(m) == INFINITY ? m : m + by, m2 < 0.f ? 0.f : m2);  // (a NaN stays one)
        }
    }
    if (s.cluster > 1) {
        gn_cluster_arrive();
        gn_cluster_wait();
    } else {
        __syncthreads();
    }
    for (int g = warp; g < groups; g += kWarps) {  // a lane per CTA of the cluster
        float2 e = make_float2(0.f, 0.f);
        float n = 0.f;
        if (lane < s.cluster) {
            e = s.cluster > 1 ? gn_remote(&sh_cta[g], lane) : sh_cta[g];
            const int64_t first = (int64_t)lane * s.share, last = first + s.share < a.t.P ? first + s.share : a.t.P;
            n = last > first ? (float)((int)(last - first) * s.per) : 0.f;
        }
        const float all = (float)(a.t.P * s.per);
        const float first = __shfl_sync(0xffffffffu, e.x, 0);
        float mean = n > 0.f ? n * (e.x - first) : 0.f;
#pragma unroll
        for (int o = kGnMaxCluster / 2; o > 0; o >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, o);
        mean = first + __shfl_sync(0xffffffffu, mean, 0) / all;
        if (mean != mean) {  // infinities: of one sign, the mean is theirs (all lanes have the same value here)
            mean = n > 0.f ? n * e.x : 0.f;
#pragma unroll
            for (int o = kGnMaxCluster / 2; o > 0; o >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, o);
            mean = __shfl_sync(0xffffffffu, mean, 0) / all;
        }
        const float d = e.x - mean;
        float m2 = n > 0.f ? __fmaf_rn(n * d, d, e.y) : 0.f;
#pragma unroll
        for (int o = kGnMaxCluster / 2; o > 0; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
        if (lane == 0) {
            const float rstd = 1.f / sqrtf(m2 / all + a.eps);
            sh_mean[g] = mean;
            sh_rstd[g] = rstd;
            if (q.rank == 0) {
                const int64_t at = q.n * a.t.G + (q.c - q.c0) / s.per + g;
                a.mean[at] = mean;
                a.rstd[at] = rstd;
            }
        }
    }
    __syncthreads();
    if (s.cluster > 1) gn_cluster_arrive();  // this CTA has read the others' sums
    if (q.active) {
        GnAffine<8> z;
        int g = q.c0 / s.per, left = (g + 1) * s.per - q.c0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (left == 0) { ++g; left = s.per; }
            --left;
            z.set(j, sh_mean[g], sh_rstd[g], a.gamma ? a.gamma[q.c + j] : 1.f, a.beta ? a.beta[q.c + j] : 0.f);
        }
        const unsigned team = 0xfu << (threadIdx.x & 28);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = q.n * a.t.P + q.first + q.ty + u * s.rows;
            float f[8], y[8];
            unpack8(v[u], f);
            if constexpr (KEEP != 0) {  // four lanes hold a group of 32 channels; the same pixel, so all four are in or none is
                uint32_t b = max_abs_bits(v[u]);
                b = max(b, __shfl_xor_sync(team, b, 1));
                b = max(b, __shfl_xor_sync(team, b, 2));
                const uint32_t byte = act8_byte(b);
                if (in[u]) {
                    *reinterpret_cast<uint2*>(a.codes + row * a.t.C + q.c) =
                        act8_codes<KEEP == 2>(f, byte, (uint64_t)(row * a.t.C + q.c), 0u, a.stream_id, a.keys);
                    if ((threadIdx.x & 3) == 0) a.scales[(uint64_t)(row * a.t.C + q.c) / kAct8Group] = (uint8_t)byte;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = act_value<ACT, kAccurate>(z.z(z.centre(f[j], j), j));
            if (in[u]) store8((E*)a.out + row * a.t.C + q.c, y);
        }
    }
    if (s.cluster > 1) gn_cluster_wait();  // the others have read this CTA's
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
    GnSlab slab;
    if (vec && p.P > 0 && (!p.codes || fused)) {
        const int u = gn_vectors(p.N, p.P, p.C, p.G, (int)size, fused, size == 4 ? 4 : 8, kGnForwardWork, sm_count, slab);
        if (u) {
            const GnArgs a = gn_args(p, gn_tiles(p.N, p.P, p.C, p.G, 8, sm_count, 1));
            launch_begin("k_gn_forward", stream);
            const cudaError_t e = with_dtype(p.dtype, [&](auto elem) {
                using E = decltype(elem);
                return with_act(p.act, [&](auto act) {
                    constexpr int A = decltype(act)::value;
                    const auto with = [&](auto vectors) {
                        constexpr int U = decltype(vectors)::value;
                        if (!fused) return launch_cluster(k_gn_forward<E, A, 0, U>, slab.ctas, slab.cluster, stream, a, slab);
                        if (p.rounding == OGQ_ROUND_RANDOM) return launch_cluster(k_gn_forward<E, A, 2, U>, slab.ctas, slab.cluster, stream, a, slab);
                        return launch_cluster(k_gn_forward<E, A, 1, U>, slab.ctas, slab.cluster, stream, a, slab);
                    };
                    if constexpr (sizeof(E) == 2) {
                        if (u == 8) return with(std::integral_constant<int, 8>{});
                    }
                    return u == 4 ? with(std::integral_constant<int, 4>{}) : with(std::integral_constant<int, 2>{});
                });
            });
            launch_end(stream);
            return e;
        }
    }
    cudaError_t e = cudaSuccess;
    if (p.codes && !fused && p.P > 0) {  // before the elements: y may be x
        Act8Forward f = {};
        f.x = p.x; f.ld_x = p.C; f.rows = p.N * p.P; f.cols = p.C;
        f.dtype = p.dtype; f.rounding = p.rounding; f.seed = p.seed; f.stream_id = p.stream_id;
        f.codes = p.codes; f.scales = p.scales;
        e = launch_act8_forward(f, sm_count, stream);
        if (e != cudaSuccess) return e;
    }
    const auto launch = [&](const char* name, auto kernel, int V, int least, GnArgs& a) {
        a = gn_args(p, gn_tiles(p.N, p.P, p.C, p.G, V, gn_wave(kernel, sm_count), least));
        if (a.t.ctas == 0) return cudaSuccess;
        if (a.t.ctas > 0x7fffffff) return cudaErrorInvalidValue;
        launch_begin(name, stream);
        const cudaError_t r = launch_pdl(kernel, (int)a.t.ctas, kThreads, 0, stream, a);
        launch_end(stream);
        return r;
    };
    GnArgs sums;
    e = with_dtype(p.dtype, [&](auto elem) {
        using E = decltype(elem);
        return vec ? launch("k_gn_moments", k_gn_moments<E, 8>, 8, kGnMinChunk, sums) : launch("k_gn_moments", k_gn_moments<E, 1>, 1, kGnMinChunk, sums);
    });
    if (e != cudaSuccess) return e;
    launch_begin("k_gn_stats", stream);
    e = launch_pdl(k_gn_stats, (int)(p.N * p.G), kThreads, 0, stream, sums);
    launch_end(stream);
    if (e != cudaSuccess) return e;
    return with_dtype(p.dtype, [&](auto elem) {
        using E = decltype(elem);
        GnArgs a;
        if (!vec) return launch("k_gn_apply", k_gn_apply<E, 1, -1, 0>, 1, 2, a);
        return with_act(p.act, [&](auto act) {
            constexpr int A = decltype(act)::value;
            if (!fused) return launch("k_gn_apply", k_gn_apply<E, 8, A, 0>, 8, 2, a);
            if (p.rounding == OGQ_ROUND_RANDOM) return launch("k_gn_apply", k_gn_apply<E, 8, A, 2>, 8, 2, a);
            return launch("k_gn_apply", k_gn_apply<E, 8, A, 1>, 8, 2, a);
        });
    });
}

}  // namespace ogq

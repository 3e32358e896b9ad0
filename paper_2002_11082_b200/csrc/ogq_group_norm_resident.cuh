// Group norm whose slabs stay on the chip: a cluster of CTAs holds one sample's values of `width` neighbouring channels (whole
// groups) in registers, so that they are read once.  Thread (tx, ty) of a CTA has the 8 channels 8 tx ... and the pixels ty, ty + rows,
// ... (at most U) of the CTA's share.  Sums over the pixels go through warps, shared memory and the cluster, in a fixed order.
#pragma once

#include "ogq_group_norm.cuh"

namespace ogq {

constexpr int kGnMaxCluster = 8;    // the portable size
constexpr int kGnMaxWidth = 512;    // channels of a slab
// Vectors per thread of an SM's CTAs, up to which a slab's pass is faster than streaming (32 x 3136 x 64 bf16: forward, 24 a thread and
// SM, 19 us against 23; backward, 28, 34 us against 24).
constexpr int kGnForwardWork = 32, kGnBackwardWork = 16;
constexpr int kGnMostCtas = 8;      // per SM: with more of them a thread takes more vectors (32 x 196 x 1024 bf16 forward: 24 us with two each, 15 with four)

struct GnSlab {
    int width;      // channels of a slab
    int wv;         // width / 8
    int rows;       // pixels side by side: kThreads / wv
    int slabs;      // of a sample
    int cluster;
    int share;      // pixels of a CTA
    int per;        // channels of a group
    int sum_rows;   // rows of partial sums in shared memory: the warps', or each row of threads'
    bool in_warp;   // lanes of a warp with the same channels are added by shuffles first (wv a power of two, at most 16)
    int64_t ctas;
};

// The slab of the smallest width that is whole groups, whole vectors, whole units of 32 where x is kept, and at least `bytes` wide;
// false where none divides C or P pixels do not fit U to a thread.
inline bool gn_slab(int64_t N, int64_t P, int64_t C, int64_t G, int size, bool keep, int U, int bytes, GnSlab& s)
{
    const int64_t per = C / G, unit = keep ? 32 : 8;
    int64_t least = unit;
    while (least % per != 0 && least <= kGnMaxWidth) least += unit;
    int64_t width = 0;
    for (int64_t w = least; w <= kGnMaxWidth && w <= C; w += least)
        if (C % w == 0 && (w * size >= bytes || w == C)) { width = w; break; }
    if (width == 0) return false;
    s.width = (int)width;
    s.wv = (int)(width / 8);
    s.rows = kThreads / s.wv;
    s.slabs = (int)(C / width);
    s.per = (int)per;
    const int64_t holds = (int64_t)s.rows * U;
    const int64_t k = (P + holds - 1) / holds;
    if (k < 1 || k > kGnMaxCluster) return false;
    s.cluster = (int)k;
    s.share = (int)((P + k - 1) / k);
    s.in_warp = s.wv <= 16 && (s.wv & (s.wv - 1)) == 0;
    s.sum_rows = s.in_warp ? kWarps : s.rows;
    s.ctas = N * s.slabs * k;
    return s.ctas <= 0x7fffffff;
}

// The fewest vectors a thread, of 2, 4 and (most = 8) 8, for which the slabs fit and are little enough work; 0: none.  Slabs of whole pairs of
// sectors, or single ones (whose other half another CTA asks for at the same time) where those hold too few pixels.
inline int gn_vectors(int64_t N, int64_t P, int64_t C, int64_t G, int size, bool keep, int most, int work, int sm_count, GnSlab& s)
{
    for (int bytes = 64; bytes >= 32; bytes /= 2)
        for (int u = 2; u <= most; u *= 2)
            if (gn_slab(N, P, C, G, size, keep, u, bytes, s) && s.ctas <= (int64_t)sm_count * kGnMostCtas &&
                s.ctas * u <= (int64_t)sm_count * work)
                return u;
    return 0;
}

__device__ __forceinline__ uint32_t gn_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// (.aligned: the lanes of a warp must come together, wherever the code before has taken them)
__device__ __forceinline__ void gn_cluster_arrive()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
}
__device__ __forceinline__ void gn_cluster_wait()
{
    __syncwarp();
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
// The float2 at `p` of this CTA's shared memory, in CTA `rank` of the cluster.
__device__ __forceinline__ float2 gn_remote(const float2* p, uint32_t rank)
{
    float2 v;
    asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %2, %3;\n\tld.shared::cluster.v2.f32 {%0, %1}, [a];\n\t}"
                 : "=f"(v.x), "=f"(v.y) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank) : "memory");
    return v;
}

// This thread's place in its slab.
struct GnSpot {
    int64_t n, c;        // sample, first channel
    int rank, tx, ty;
    int64_t first, last; // pixels of the CTA
    int c0;              // first channel of the thread in the slab
    bool active;
};
__device__ __forceinline__ GnSpot gn_spot(const GnTiles& t, const GnSlab& s)
{
    GnSpot q;
    q.rank = (int)gn_rank();
    const int slab = (int)(blockIdx.x / (unsigned)s.cluster);
    q.n = slab / s.slabs;
    q.ty = threadIdx.x / (unsigned)s.wv;
    q.tx = threadIdx.x - q.ty * s.wv;
    q.c0 = q.tx * 8;
    q.c = (int64_t)(slab - (int)q.n * s.slabs) * s.width + q.c0;
    q.active = q.ty < s.rows;
    q.first = (int64_t)q.rank * s.share;
    q.last = q.first + s.share < t.P ? q.first + s.share : t.P;
    return q;
}

// Leaves this CTA's partial sums of the thread's 8 channels in sh[row][channel of the slab], sum_rows rows.
template <class Tv>
__device__ __forceinline__ void gn_put_sums(const GnSlab& s, const GnSpot& q, Tv (&v)[8], Tv* sh, int pitch)
{
    if (s.in_warp) {
        for (int o = 16; o >= s.wv; o >>= 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (sizeof(Tv) == 8) {
                    v[j].x += __shfl_xor_sync(0xffffffffu, v[j].x, o);
                    v[j].y += __shfl_xor_sync(0xffffffffu, v[j].y, o);
                } else {
                    v[j] += __shfl_xor_sync(0xffffffffu, v[j], o);
                }
            }
        }
        if ((int)(threadIdx.x & 31) < s.wv) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sh[(threadIdx.x >> 5) * pitch + q.c0 + j] = v[j];
        }
    } else if (q.active) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sh[q.ty * pitch + q.c0 + j] = v[j];
    }
}

// A cluster launch that may begin while the kernel before it still runs.
template <class... Params, class... Args>
inline cudaError_t launch_cluster(void (*kernel)(Params...), int64_t ctas, int cluster, cudaStream_t stream, Args... args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

}  // namespace ogq

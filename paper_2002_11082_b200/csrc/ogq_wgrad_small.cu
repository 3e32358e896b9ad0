// Weight and bias gradient from an input kept in 8 bits, for few weights and rows: one launch whatever the type and the addresses.
//   A tile of 32 x 32 weights per cluster of CTAs, which share the rows; 64 rows at a time in shared memory as fp32, the next ones already asked
// for; fp32 multiply-adds (the products of 24 and 8 bits are rounded with the addition).  The cluster's sums are added in the order of its CTAs.
//   Bound by latency: launch, two rounds of loads, a cluster barrier.
#include "ogq_act8.cuh"
#include "ogq_group_norm_resident.cuh"
#include "ogq_internal.h"

namespace ogq {

constexpr int kWsTile = 32, kWsChunk = 64, kWsEach = kWsChunk / kWarps;

struct WsArgs {
    const void* dy; int64_t ld_dy;
    const int8_t* codes; const uint8_t* scales;
    int64_t rows, cols, out_cols;
    int groups, tiles_i, cluster;
    int share;  // rows of a CTA
    float* dw; float* db;
    bool accumulate;
};

template <class E>
__global__ void __launch_bounds__(kThreads) k_wgrad_small(const __grid_constant__ WsArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float sdy[kWsChunk][kWsTile], sx[kWsChunk][kWsTile];
    __shared__ float2 part[kWsTile][kWsTile / 2], bias_part[kWsTile / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)gn_rank();
    const uint32_t tile = blockIdx.x / (uint32_t)a.cluster, to = tile / (uint32_t)a.tiles_i, ti = tile - to * (uint32_t)a.tiles_i;
    const int64_t o0 = (int64_t)to * kWsTile, i0 = (int64_t)ti * kWsTile;
    const int64_t begin = (int64_t)rank * a.share, end = begin + a.share < a.rows ? begin + a.share : a.rows;
    const bool has_o = o0 + lane < a.out_cols, has_i = i0 + lane < a.cols;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;

    E dy[kWsEach];
    int8_t code[kWsEach];
    uint32_t scale[kWsEach];
    const auto load = [&](int64_t t0) {
#pragma unroll
        for (int j = 0; j < kWsEach; ++j) {
            const int64_t t = t0 + warp + kWarps * j;
            if (t < end) {
                if (has_o) dy[j] = ((const E*)a.dy)[t * a.ld_dy + o0 + lane];
                if (has_i) {
                    code[j] = a.codes[t * a.cols + i0 + lane];
                    scale[j] = a.scales[t * a.groups + ti];
                }
            }
        }
    };
    float acc[2][2] = {{0.f, 0.f}, {0.f, 0.f}}, bias = 0.f;
    load(begin);
    for (int64_t t0 = begin; t0 < end; t0 += kWsChunk) {
#pragma unroll
        for (int j = 0; j < kWsEach; ++j) {
            const bool in = t0 + warp + kWarps * j < end;
            sdy[warp + kWarps * j][lane] = in && has_o ? load1(&dy[j]) : 0.f;
            sx[warp + kWarps * j][lane] = in && has_i ? (float)code[j] * act8_unit(scale[j]) : 0.f;
        }
        __syncthreads();
        load(t0 + kWsChunk);
        const int n = (int)(end - t0 < kWsChunk ? end - t0 : kWsChunk);
#pragma unroll 8
        for (int k = 0; k < n; ++k) {
            const float2 d = *reinterpret_cast<const float2*>(&sdy[k][ty * 2]), x = *reinterpret_cast<const float2*>(&sx[k][tx * 2]);
            acc[0][0] = __fmaf_rn(d.x, x.x, acc[0][0]);
            acc[0][1] = __fmaf_rn(d.x, x.y, acc[0][1]);
            acc[1][0] = __fmaf_rn(d.y, x.x, acc[1][0]);
            acc[1][1] = __fmaf_rn(d.y, x.y, acc[1][1]);
        }
        if (ti == 0 && warp == 0 && a.db)
#pragma unroll 8
            for (int k = 0; k < n; ++k) bias = __fadd_rn(bias, sdy[k][lane]);
        __syncthreads();
    }
    const auto put = [&](int64_t o, int64_t i, float v) {
        if (o >= a.out_cols || i >= a.cols) return;
        float* w = a.dw + o * a.cols + i;
        *w = a.accumulate ? *w + v : v;
    };
    const auto put_bias = [&](float v) {
        if (has_o) a.db[o0 + lane] = a.accumulate ? a.db[o0 + lane] + v : v;
    };
    const bool has_bias = ti == 0 && a.db;
    if (a.cluster == 1) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            put(o0 + ty * 2 + q, i0 + tx * 2, acc[q][0]);
            put(o0 + ty * 2 + q, i0 + tx * 2 + 1, acc[q][1]);
        }
        if (has_bias && warp == 0) put_bias(bias);
        return;
    }
    part[ty * 2][tx] = make_float2(acc[0][0], acc[0][1]);
    part[ty * 2 + 1][tx] = make_float2(acc[1][0], acc[1][1]);
    if (warp == 0) reinterpret_cast<float*>(bias_part)[lane] = bias;
    gn_cluster_arrive();
    gn_cluster_wait();
    const int mine = kWsTile / a.cluster;  // rows of the tile that this CTA adds up
    if (ty < mine) {
        const int r = rank * mine + ty;
        float2 s = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < a.cluster; ++c) {
            const float2 v = gn_remote(&part[r][tx], c);
            s.x += v.x;
            s.y += v.y;
        }
        put(o0 + r, i0 + tx * 2, s.x);
        put(o0 + r, i0 + tx * 2 + 1, s.y);
    }
    if (has_bias && rank == 0 && warp == 7) {
        float s = 0.f;
        for (int c = 0; c < a.cluster; ++c) {
            const float2 v = gn_remote(&bias_part[lane >> 1], c);
            s += lane & 1 ? v.y : v.x;
        }
        put_bias(s);
    }
    gn_cluster_arrive();
    gn_cluster_wait();  // the others have read this CTA's
}

// Measured, us, this kernel and the tensor cores' (more_launches: operands are laid out first, or the bias has a kernel of its own):
//   bf16, one launch   32 x 64 x 64: 3.3 and 5.1;  128 x 512 x 512: 7.5 and 8.2;  500 x 256 x 256: 8.8 and 10.3;
//                      beyond: 32 x 1024 x 1024: 8.7 and 7.9;  2000 x 32 x 32: 10.2 and 8.9
//   more launches      32 x 512 x 512 fp32: 5.3 and 12.4;  32 x 1024 x 1024 fp32: 8.7 and 12.6;  2000 x 32 x 32 bf16 with bias: 11.7 and 14.6;
//                      beyond: 4 x 2880 x 2880 fp32: 35.9 and 19.8
bool act8_wgrad_is_small(const Wgrad8& p, bool more_launches)
{
    const int64_t rows = more_launches ? 2048 : 512, weights = more_launches ? 1 << 20 : 1 << 18;
    if (p.rows <= 0 || p.cols <= 0 || p.rows > rows || p.cols > weights || p.out_cols > weights || p.cols * p.out_cols > weights) return false;
    return p.rows * p.cols * p.out_cols <= (int64_t)1 << 25;
}

cudaError_t launch_act8_wgrad_small(const Wgrad8& p, cudaStream_t stream)
{
    WsArgs a = {p.dy, p.ld_dy, p.codes, p.scales, p.rows, p.cols, p.out_cols, (int)act8_groups(p.cols), 0, 1, 0, p.dw, p.db, p.accumulate != 0};
    a.tiles_i = (int)((p.cols + kWsTile - 1) / kWsTile);
    while (a.cluster < 8 && p.rows > 128 * a.cluster) a.cluster *= 2;
    a.share = (int)((p.rows + a.cluster - 1) / a.cluster);
    const int64_t ctas = (p.out_cols + kWsTile - 1) / kWsTile * a.tiles_i * a.cluster;
    launch_begin("k_wgrad_small", stream);
    const cudaError_t e = with_dtype(p.dtype, [&](auto elem) { return launch_cluster(k_wgrad_small<decltype(elem)>, ctas, a.cluster, stream, a); });
    launch_end(stream);
    return e;
}

}  // namespace ogq

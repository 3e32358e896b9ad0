// Weight and bias gradient of a linear layer from its input kept in 8 bits: dW = dy^T x^, db = sum of dy's rows.
#include "ogq_act8.cuh"
#include "ogq_internal.h"

namespace ogq {

struct WgArgs {
    const void* dy; int64_t ld_dy;
    const int8_t* codes; const uint8_t* scales;
    int64_t rows, cols, out_cols;
    float* dw; float* db;
    bool accumulate;
};

// A tile of 32 x 32 weights per CTA, 32 rows at a time.
template <class E>
__global__ void __launch_bounds__(kThreads) k_wgrad_any(const __grid_constant__ WgArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float dy[32][33], x[32][33];
    const int64_t tiles = a.cols > 0 ? (a.cols + 31) / 32 : 1;  // no columns: the bias alone
    const int64_t o0 = blockIdx.x / tiles * 32, i0 = (blockIdx.x - o0 / 32 * tiles) * 32;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, bias[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t t0 = 0; t0 < a.rows; t0 += 32) {
        for (int k = ty; k < 32; k += 8) {
            const int64_t t = t0 + k;
            dy[k][tx] = t < a.rows && o0 + tx < a.out_cols ? load1((const E*)a.dy + t * a.ld_dy + o0 + tx) : 0.f;
            x[k][tx] = t < a.rows && i0 + tx < a.cols
                           ? (float)a.codes[t * a.cols + i0 + tx] * act8_unit(a.scales[t * act8_groups(a.cols) + (i0 + tx) / kAct8Group]) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 32; ++k) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[j] = __fmaf_rn(dy[k][ty * 4 + j], x[k][tx], acc[j]);
                bias[j] += dy[k][ty * 4 + j];
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t o = o0 + ty * 4 + j;
        if (o >= a.out_cols) break;
        if (i0 + tx < a.cols) {
            float* w = a.dw + o * a.cols + i0 + tx;
            *w = a.accumulate ? *w + acc[j] : acc[j];
        }
        if (a.db && i0 == 0 && tx == 0) a.db[o] = a.accumulate ? a.db[o] + bias[j] : bias[j];
    }
}

size_t ws_bytes_act8_wgrad(int64_t, int64_t, int64_t, int, int) { return 0; }

cudaError_t launch_act8_wgrad(const Wgrad8& p, int, cudaStream_t stream)
{
    WgArgs a = {p.dy, p.ld_dy, p.codes, p.scales, p.rows, p.cols, p.out_cols, p.dw, p.db, p.accumulate != 0};
    const int64_t tiles = p.cols > 0 ? (p.cols + 31) / 32 : 1;
    const int64_t ctas = tiles * ((p.out_cols + 31) / 32);
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    launch_begin("k_wgrad", stream);
    const cudaError_t e = with_dtype(p.dtype, [&](auto elem) {
        return launch_pdl(k_wgrad_any<decltype(elem)>, (int)ctas, kThreads, 0, stream, a);
    });
    launch_end(stream);
    return e;
}

}  // namespace ogq

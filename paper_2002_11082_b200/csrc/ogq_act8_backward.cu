// Activations kept in 8 bits: the decoder, and the backward pass of the activation function from its kept inputs.
//   dx = dy f'(x^) [up^],  dup = dy f(x^)
// Bound by memory: dy and 33/32 bytes per kept element read once, the gradients written once.
#include "ogq_act8.cuh"
#include "ogq_internal.h"

namespace ogq {

struct BwdArgs {
    const void* dy;  // null: decode
    void* dx; void* dup;
    const int8_t* codes; const int8_t* up_codes;
    const uint8_t* scales; const uint8_t* up_scales;
    int64_t ld_dy, ld_dx, ld_dup, cols;
    uint32_t groups;      // of a row
    uint32_t all_groups;  // of the matrix
    int act;              // of the kernel of single elements
};

// Any sizes, strides and addresses: a warp per group, a lane per element.
template <class E, bool GATED>
__global__ void __launch_bounds__(kThreads) k_act8_backward_any(const __grid_constant__ BwdArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    const int lane = threadIdx.x & 31;
    const uint32_t warps = gridDim.x * kWarps;
    for (uint32_t g = blockIdx.x * kWarps + (threadIdx.x >> 5); g < a.all_groups; g += warps) {
        const uint32_t row = g / a.groups;
        const int64_t col = (int64_t)(g - row * a.groups) * kAct8Group + lane;
        if (col >= a.cols) continue;
        const int64_t at = (int64_t)row * a.cols + col;
        const float x = (float)a.codes[at] * act8_unit(a.scales[g]);
        float dx = x;
        if (a.dy) {
            const float dy = load1((const E*)a.dy + row * a.ld_dy + col);
            float f = x, slope = 1.f;
            switch (a.act) {
                case OGQ_ACT_RELU: f = act_both<OGQ_ACT_RELU, kAccurate>(x, slope); break;
                case OGQ_ACT_SILU: f = act_both<OGQ_ACT_SILU, kAccurate>(x, slope); break;
                case OGQ_ACT_GELU: f = act_both<OGQ_ACT_GELU, kAccurate>(x, slope); break;
            }
            dx = dy;
            if (GATED) {
                dx *= (float)a.up_codes[at] * act8_unit(a.up_scales[g]);
                store1((E*)a.dup + row * a.ld_dup + col, dy * f);
            }
            dx *= slope;
        }
        store1((E*)a.dx + row * a.ld_dx + col, dx);
    }
}

cudaError_t launch_act8_backward(const Act8Backward& p, int sm_count, cudaStream_t stream)
{
    BwdArgs a = {};
    a.dy = p.dy; a.dx = p.dx; a.dup = p.dup;
    a.codes = p.codes; a.up_codes = p.up_codes; a.scales = p.scales; a.up_scales = p.up_scales;
    a.ld_dy = p.ld_dy; a.ld_dx = p.ld_dx; a.ld_dup = p.ld_dup; a.cols = p.cols;
    a.groups = (uint32_t)act8_groups(p.cols);
    a.all_groups = (uint32_t)(p.rows * a.groups);
    a.act = p.act;
    const int64_t want = ((int64_t)a.all_groups + kWarps - 1) / kWarps;
    const int ctas = (int)(want < (int64_t)sm_count * 8 ? want : (int64_t)sm_count * 8);
    launch_begin(p.dy ? "k_act8_backward" : "k_act8_decode", stream);
    const cudaError_t e = with_dtype(p.dtype, [&](auto elem) {
        using E = decltype(elem);
        return with_bool(p.dup != nullptr, [&](auto gated) {
            return launch_pdl(k_act8_backward_any<E, decltype(gated)::value>, ctas, kThreads, 0, stream, a);
        });
    });
    launch_end(stream);
    return e;
}

}  // namespace ogq

// Activations kept in 8 bits: the encoder, and the activation function that keeps its inputs.
//   unit 2^e of a group of 32 columns, e the smallest integer with max|x| <= 127 * 2^e; code = x / 2^e rounded.
//   y = f(x) [* up]
// Bound by memory: x read once, y and 33/32 bytes per element written once.
#include "ogq_act8.cuh"
#include "ogq_internal.h"

namespace ogq {

struct FwdArgs {
    const void* x; const void* up;
    void* y;
    int8_t* codes; int8_t* up_codes;
    uint8_t* scales; uint8_t* up_scales;
    int64_t ld_x, ld_up, ld_y, cols;
    uint32_t groups;      // of a row
    uint32_t all_groups;  // of the matrix
    uint32_t stream_id;
    int act;              // of the kernel of single elements
    bool random;
    PhiloxKeys keys;
};

// Any sizes, strides and addresses: a warp per group, a lane per element.
template <class E, bool GATED>
__global__ void __launch_bounds__(kThreads) k_act8_forward_any(const __grid_constant__ FwdArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    const int lane = threadIdx.x & 31;
    const uint32_t warps = gridDim.x * kWarps;
    for (uint32_t g = blockIdx.x * kWarps + (threadIdx.x >> 5); g < a.all_groups; g += warps) {
        const uint32_t row = g / a.groups;
        const int64_t col = (int64_t)(g - row * a.groups) * kAct8Group + lane;
        const bool in = col < a.cols;
        const int64_t at = (int64_t)row * a.cols + col;
        float v = 0.f, u = 0.f;
        if (in) {
            v = load1((const E*)a.x + row * a.ld_x + col);
            if (GATED) u = load1((const E*)a.up + row * a.ld_up + col);
        }
#pragma unroll
        for (int k = 0; k < (GATED ? 2 : 1); ++k) {
            const float w = k ? u : v;
            const uint32_t byte = act8_byte(__reduce_max_sync(0xffffffffu, abs_bits(w)));
            uint32_t code;
            if (a.random) {
                const uint64_t block = (uint64_t)at / 4;
                const uint4 r = philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), (uint32_t)k, a.stream_id, a.keys);
                const uint32_t i = (uint32_t)at & 3u;
                code = act8_code_random(w, byte, i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w);
            } else {
                code = act8_code(w, byte);
            }
            if (in) (k ? a.up_codes : a.codes)[at] = (int8_t)(uint8_t)code;
            if (lane == 0) (k ? a.up_scales : a.scales)[g] = (uint8_t)byte;
        }
        if (in && a.y) {
            float y = v;
            switch (a.act) {
                case OGQ_ACT_RELU: y = act_value<OGQ_ACT_RELU, kAccurate>(v); break;
                case OGQ_ACT_SILU: y = act_value<OGQ_ACT_SILU, kAccurate>(v); break;
                case OGQ_ACT_GELU: y = act_value<OGQ_ACT_GELU, kAccurate>(v); break;
            }
            if (GATED) y *= u;
            store1((E*)a.y + row * a.ld_y + col, y);
        }
    }
}

cudaError_t launch_act8_forward(const Act8Forward& p, int sm_count, cudaStream_t stream)
{
    FwdArgs a = {};
    a.x = p.x; a.up = p.up; a.y = p.y;
    a.codes = p.codes; a.up_codes = p.up_codes; a.scales = p.scales; a.up_scales = p.up_scales;
    a.ld_x = p.ld_x; a.ld_up = p.ld_up; a.ld_y = p.ld_y; a.cols = p.cols;
    a.groups = (uint32_t)act8_groups(p.cols);
    a.all_groups = (uint32_t)(p.rows * a.groups);
    a.stream_id = p.stream_id;
    a.act = p.act;
    a.random = p.rounding == OGQ_ROUND_RANDOM;
    a.keys = philox_round_keys((uint32_t)p.seed, (uint32_t)(p.seed >> 32));
    const int64_t want = ((int64_t)a.all_groups + kWarps - 1) / kWarps;
    const int ctas = (int)(want < (int64_t)sm_count * 8 ? want : (int64_t)sm_count * 8);
    launch_begin("k_act8_forward", stream);
    const cudaError_t e = with_dtype(p.dtype, [&](auto elem) {
        using E = decltype(elem);
        return with_bool(p.up != nullptr, [&](auto gated) {
            return launch_pdl(k_act8_forward_any<E, decltype(gated)::value>, ctas, kThreads, 0, stream, a);
        });
    });
    launch_end(stream);
    return e;
}

}  // namespace ogq

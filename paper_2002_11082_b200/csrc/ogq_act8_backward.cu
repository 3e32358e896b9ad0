// Activations kept in 8 bits: the decoder, and the backward pass of the activation function from its kept inputs.
//   dx = dy f'(x^) [up^],  dup = dy f(x^)
// Bound by memory: dy and 33/32 bytes per kept element read once, the gradients written once.  16,384 x 4096 bf16 decoded: 33 us, 6.2 TB/s; gated
// SiLU on 8192 x 8192 bf16: 84 us, 6.4 TB/s.  GELU in 16 bits is bound by its 37 instructions an element.
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
    uint32_t div_mul, div_shift;  // g / groups = hi(g * div_mul) >> div_shift
};

// Any sizes, strides and addresses: eight lanes a group, elements l, l + 8, l + 16, l + 24 of it for lane l, two groups a lane under way.
template <class E, int ACT, bool GATED, bool DECODE>
__global__ void __launch_bounds__(kThreads) k_act8_backward_any(const __grid_constant__ BwdArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    constexpr int kUnits = 2;
    constexpr uint32_t kTeams = kThreads / 8;
    const int l = threadIdx.x & 7;
    const uint32_t team = threadIdx.x >> 3;
    for (uint32_t g0 = blockIdx.x * (kTeams * kUnits) + team; g0 < a.all_groups; g0 += gridDim.x * (kTeams * kUnits)) {
        float v[kUnits][4], u[kUnits][4], d[kUnits][4], unit[kUnits], up_unit[kUnits];
        uint32_t row[kUnits];
        int col[kUnits], n[kUnits];  // first column, how many of this lane's four elements
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const uint32_t g = g0 + k * kTeams;
            row[k] = act8_row(a, g);
            col[k] = (int)(g - row[k] * a.groups) * kAct8Group + l;
            const int left = (int)a.cols - col[k];
            n[k] = g >= a.all_groups || left <= 0 ? 0 : left >= 25 ? 4 : (left + 7) >> 3;
            const int64_t at = (int64_t)row[k] * a.cols + col[k];
            if (n[k] > 0) {
                unit[k] = act8_unit(a.scales[g]);
                if (GATED) up_unit[k] = act8_unit(a.up_scales[g]);
            }
            const E* dy = (const E*)a.dy + row[k] * a.ld_dy + col[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e < n[k]) {
                    v[k][e] = (float)a.codes[at + 8 * e];
                    if (GATED) u[k][e] = (float)a.up_codes[at + 8 * e];
                    if (!DECODE) d[k][e] = load1(dy + 8 * e);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            E* out = (E*)a.dx + row[k] * a.ld_dx + col[k];
            E* dup = (E*)a.dup + row[k] * a.ld_dup + col[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = v[k][e] * unit[k];
                float dx = x;
                if constexpr (!DECODE) {
                    float slope;
                    const float f = act_both<ACT, kAccurate>(x, slope);
                    dx = d[k][e] * slope;
                    if (GATED) {
                        dx *= u[k][e] * up_unit[k];
                        if (e < n[k]) store1(dup + 8 * e, d[k][e] * f);
                    }
                }
                if (e < n[k]) store1(out + 8 * e, dx);
            }
        }
    }
}

// Rows of whole eights of elements on 16-byte boundaries: eight elements a thread at a time, kUnits such pieces under way.
template <class E, int ACT, bool GATED, bool DECODE>
__global__ void __launch_bounds__(kThreads) k_act8_backward(const __grid_constant__ BwdArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    constexpr int kUnits = GATED || sizeof(E) == 4 ? 2 : 4;
    const uint32_t team = threadIdx.x >> 2;
    const int part = threadIdx.x & 3;
    const uint32_t stride = kThreads / 4;
    for (uint32_t g0 = blockIdx.x * (stride * kUnits) + team; g0 < a.all_groups; g0 += gridDim.x * (stride * kUnits)) {
        Raw8<E> dy[DECODE ? 1 : kUnits];
        uint2 x[kUnits], u[GATED ? kUnits : 1];
        uint32_t sx[kUnits], su[GATED ? kUnits : 1];
        int64_t row[kUnits], col[kUnits];
        bool in[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const uint32_t g = g0 + k * stride;
            const uint32_t r = act8_row(a, g);
            row[k] = r;
            col[k] = (int64_t)(g - r * a.groups) * kAct8Group + part * 8;
            in[k] = g < a.all_groups && col[k] < a.cols;
            if (in[k]) {
                const int64_t at = row[k] * a.cols + col[k];
                x[k] = *reinterpret_cast<const uint2*>(a.codes + at);
                sx[k] = a.scales[g];
                if constexpr (GATED) {
                    u[k] = *reinterpret_cast<const uint2*>(a.up_codes + at);
                    su[k] = a.up_scales[g];
                }
                if constexpr (!DECODE) dy[k] = load_raw8((const E*)a.dy + row[k] * a.ld_dy + col[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            if (!in[k]) continue;
            float v[8], d[8], w[8];
            act8_values(x[k], act8_unit(sx[k]), v);
            if constexpr (DECODE) {
                store8((E*)a.dx + row[k] * a.ld_dx + col[k], v);
            } else {
                unpack8(dy[k], d);
                if constexpr (GATED) {
                    float dup[8];
                    act8_values(u[k], act8_unit(su[k]), w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float slope;
                        dup[j] = __fmul_rn(d[j], act_both<ACT, kAccurate>(v[j], slope));
                        d[j] = __fmul_rn(__fmul_rn(d[j], slope), w[j]);  // (dy up^ alone may be infinite where the slope is 0)
                    }
                    store8((E*)a.dup + row[k] * a.ld_dup + col[k], dup);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] = __fmul_rn(d[j], act_slope<ACT, kAccurate>(v[j]));
                }
                store8((E*)a.dx + row[k] * a.ld_dx + col[k], d);
            }
        }
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
    const size_t size = p.dtype == OGQ_F32 ? 4 : 2;
    const auto whole = [&](const void* q, int64_t ld) { return ((uintptr_t)q & 15) == 0 && ld * size % 16 == 0; };
    const bool vec = p.cols % 8 == 0 && whole(p.dx, p.ld_dx) && ((uintptr_t)p.codes & 7) == 0 && (!p.dy || whole(p.dy, p.ld_dy)) &&
                     (!p.dup || (whole(p.dup, p.ld_dup) && ((uintptr_t)p.up_codes & 7) == 0));
    if (vec && p.cols % kAct8Group == 0 && p.ld_dx == p.cols && (!p.dy || p.ld_dy == p.cols) && (!p.dup || p.ld_dup == p.cols)) {
        a.groups = a.all_groups;  // one long row
        a.cols = p.rows * p.cols;
    }
    act8_divisor(a.groups, a.div_mul, a.div_shift);
    launch_begin(p.dy ? "k_act8_backward" : "k_act8_decode", stream);
    cudaError_t e;
    if (vec) {
        const int64_t per = kThreads / 4 * (p.dup || size == 4 ? 2 : 4);
        const int64_t want = ((int64_t)a.all_groups + per - 1) / per;
        const int ctas = (int)(want < (int64_t)sm_count * kAct8Ctas ? want : (int64_t)sm_count * kAct8Ctas);
        e = with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            if (!p.dy) return launch_pdl(k_act8_backward<E, OGQ_ACT_NONE, false, true>, ctas, kThreads, 0, stream, a);
            return with_bool(p.dup != nullptr, [&](auto gated) {
                return with_act(p.act, [&](auto act) {
                    return launch_pdl(k_act8_backward<E, decltype(act)::value, decltype(gated)::value, false>, ctas, kThreads, 0, stream, a);
                });
            });
        });
    } else {
        const int64_t want = ((int64_t)a.all_groups + kThreads / 4 - 1) / (kThreads / 4);
        const int ctas = (int)(want < (int64_t)sm_count * kAct8Ctas ? want : (int64_t)sm_count * kAct8Ctas);
        e = with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            if (!p.dy) return launch_pdl(k_act8_backward_any<E, OGQ_ACT_NONE, false, true>, ctas, kThreads, 0, stream, a);
            return with_bool(p.dup != nullptr, [&](auto gated) {
                return with_act(p.act, [&](auto act) {
                    return launch_pdl(k_act8_backward_any<E, decltype(act)::value, decltype(gated)::value, false>, ctas, kThreads, 0, stream, a);
                });
            });
        });
    }
    launch_end(stream);
    return e;
}

}  // namespace ogq

// Activations kept in 8 bits: the encoder, and the activation function that keeps its inputs.
//   unit 2^e of a group of 32 columns, e the smallest integer with max|x| <= 127 * 2^e; code = x / 2^e rounded.
//   y = f(x) [* up]
// Bound by memory: x read once, y and 33/32 bytes per element written once.  16,384 x 4096 bf16 encoded: 35 us, 5.8 TB/s; gated SiLU on
// 8192 x 8192 bf16: 90 us, 6.0 TB/s (copy 6.5).
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
    uint32_t div_mul, div_shift;  // g / groups = hi(g * div_mul) >> div_shift
    bool random;
    PhiloxKeys keys;
};

// Any sizes, strides and addresses: eight lanes a group, elements l, l + 8, l + 16, l + 24 of it for lane l, two groups a lane under way.
// (A warp per group and a lane per element spent 70 instructions on 32 elements: 4099 x 1001 fp16 11 us.)
template <class E, int ACT, bool GATED>
__global__ void __launch_bounds__(kThreads) k_act8_forward_any(const __grid_constant__ FwdArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    constexpr int kUnits = 2;
    constexpr uint32_t kTeams = kThreads / 8;
    const int l = threadIdx.x & 7;
    const uint32_t team = threadIdx.x >> 3;
    for (uint32_t g0 = blockIdx.x * (kTeams * kUnits) + team; __any_sync(0xffffffffu, g0 < a.all_groups); g0 += gridDim.x * (kTeams * kUnits)) {
        float v[kUnits][4], u[kUnits][4];
        uint32_t row[kUnits];
        int col[kUnits], n[kUnits];  // first column, how many of this lane's four elements
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const uint32_t g = g0 + k * kTeams;
            row[k] = act8_row(a, g);
            col[k] = (int)(g - row[k] * a.groups) * kAct8Group + l;
            const int left = (int)a.cols - col[k];
            n[k] = g >= a.all_groups || left <= 0 ? 0 : left >= 25 ? 4 : (left + 7) >> 3;
            const E* x = (const E*)a.x + row[k] * a.ld_x + col[k];
            const E* up = (const E*)a.up + row[k] * a.ld_up + col[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[k][e] = e < n[k] ? load1(x + 8 * e) : 0.f;
                if (GATED) u[k][e] = e < n[k] ? load1(up + 8 * e) : 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int64_t at = (int64_t)row[k] * a.cols + col[k];
#pragma unroll
            for (int h = 0; h < (GATED ? 2 : 1); ++h) {
                const float(&w)[4] = h ? u[k] : v[k];
                uint32_t m = max(max(abs_bits(w[0]), abs_bits(w[1])), max(abs_bits(w[2]), abs_bits(w[3])));
#pragma unroll
                for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                const uint32_t byte = act8_byte(m);
                int8_t* to = (h ? a.up_codes : a.codes) + at;
                if (a.random) {
#pragma unroll 1
                    for (int e = 0; e < n[k]; ++e) {
                        const uint64_t i = (uint64_t)at + 8 * e;
                        const uint4 r = philox4x32_10((uint32_t)(i / 4), (uint32_t)(i / 4 >> 32), (uint32_t)h, a.stream_id, a.keys);
                        const uint32_t q = (uint32_t)i & 3u;
                        const float z = e == 0 ? w[0] : e == 1 ? w[1] : e == 2 ? w[2] : w[3];
                        to[8 * e] = (int8_t)(uint8_t)act8_code_random(z, byte, q == 0 ? r.x : q == 1 ? r.y : q == 2 ? r.z : r.w);
                    }
                } else if (byte >= kAct8MaxByte) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < n[k]) to[8 * e] = (int8_t)(uint8_t)act8_code(w[e], byte);
                } else {
                    const float inv = act8_inverse_unit(byte);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < n[k]) to[8 * e] = (int8_t)(uint8_t)__float_as_uint(__fmaf_rn(w[e], inv, 12582912.f));
                }
                if (l == 0 && n[k] > 0) (h ? a.up_scales : a.scales)[g0 + k * kTeams] = (uint8_t)byte;
            }
            if (a.y) {
                E* y = (E*)a.y + row[k] * a.ld_y + col[k];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float z = act_value<ACT, kAccurate>(v[k][e]);
                    if (GATED) z = __fmul_rn(z, u[k][e]);
                    if (e < n[k]) store1(y + 8 * e, z);
                }
            }
        }
    }
}

// Rows of whole eights of elements on 16-byte boundaries: four lanes hold a group, eight elements each, and a thread has kUnits
// pieces of groups under way: 16 KB a CTA requested at once, 8 KB each of x and up with a gate.
template <class E, int ACT, bool GATED, bool RANDOM, bool HAS_Y>
__global__ void __launch_bounds__(kThreads) k_act8_forward(const __grid_constant__ FwdArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr bool kAccurate = sizeof(E) == 4;
    constexpr int kUnits = GATED || sizeof(E) == 4 ? 2 : 4;
    const uint32_t team = threadIdx.x >> 2;
    const int part = threadIdx.x & 3;
    const uint32_t stride = kThreads / 4;
    for (uint32_t g0 = blockIdx.x * (stride * kUnits) + team; __any_sync(0xffffffffu, g0 < a.all_groups); g0 += gridDim.x * (stride * kUnits)) {
        Raw8<E> x[kUnits], u[GATED ? kUnits : 1];
        int64_t row[kUnits], col[kUnits];
        bool in[kUnits];
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const uint32_t g = g0 + k * stride;
            const uint32_t r = act8_row(a, g);
            row[k] = r;
            col[k] = (int64_t)(g - r * a.groups) * kAct8Group + part * 8;
            in[k] = g < a.all_groups && col[k] < a.cols;
            x[k] = in[k] ? load_raw8((const E*)a.x + row[k] * a.ld_x + col[k]) : zero_raw8<E>();
            if constexpr (GATED) u[k] = in[k] ? load_raw8((const E*)a.up + row[k] * a.ld_up + col[k]) : zero_raw8<E>();
        }
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const uint32_t g = g0 + k * stride;
            const int64_t at = row[k] * a.cols + col[k];
            float v[8], w[8];
            unpack8(x[k], v);
            if constexpr (GATED) unpack8(u[k], w);
#pragma unroll
            for (int h = 0; h < (GATED ? 2 : 1); ++h) {
                const float(&z)[8] = h ? w : v;
                uint32_t m = max_abs_bits(h ? u[GATED ? k : 0] : x[k]);
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                const uint32_t byte = act8_byte(m);
                const uint2 c = act8_codes<RANDOM>(z, byte, (uint64_t)at, (uint32_t)h, a.stream_id, a.keys);
                if (in[k]) {
                    *reinterpret_cast<uint2*>((h ? a.up_codes : a.codes) + at) = c;
                    if (part == 0) (h ? a.up_scales : a.scales)[g] = (uint8_t)byte;
                }
            }
            if constexpr (HAS_Y) {
                if (in[k]) {
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        y[j] = act_value<ACT, kAccurate>(v[j]);
                        if constexpr (GATED) y[j] = __fmul_rn(y[j], w[j]);
                    }
                    store8((E*)a.y + row[k] * a.ld_y + col[k], y);
                }
            }
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
    a.random = p.rounding == OGQ_ROUND_RANDOM;
    a.keys = philox_round_keys((uint32_t)p.seed, (uint32_t)(p.seed >> 32));
    const size_t size = p.dtype == OGQ_F32 ? 4 : 2;
    const auto whole = [&](const void* q, int64_t ld) { return ((uintptr_t)q & 15) == 0 && ld * size % 16 == 0; };
    const bool vec = p.cols % 8 == 0 && whole(p.x, p.ld_x) && ((uintptr_t)p.codes & 7) == 0 && (!p.y || whole(p.y, p.ld_y)) &&
                     (!p.up || (whole(p.up, p.ld_up) && ((uintptr_t)p.up_codes & 7) == 0));
    if (vec && p.cols % kAct8Group == 0 && p.ld_x == p.cols && (!p.y || p.ld_y == p.cols) && (!p.up || p.ld_up == p.cols)) {
        a.groups = a.all_groups;  // one long row
        a.cols = p.rows * p.cols;
    }
    act8_divisor(a.groups, a.div_mul, a.div_shift);
    launch_begin("k_act8_forward", stream);
    cudaError_t e;
    if (vec) {
        const int64_t per = kThreads / 4 * (p.up || size == 4 ? 2 : 4);
        const int64_t want = ((int64_t)a.all_groups + per - 1) / per;
        const int ctas = (int)(want < (int64_t)sm_count * kAct8Ctas ? want : (int64_t)sm_count * kAct8Ctas);
        e = with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            return with_bool(a.random, [&](auto random) {
                constexpr bool R = decltype(random)::value;
                if (!p.y) return launch_pdl(k_act8_forward<E, OGQ_ACT_NONE, false, R, false>, ctas, kThreads, 0, stream, a);
                return with_bool(p.up != nullptr, [&](auto gated) {
                    return with_act(p.act, [&](auto act) {
                        return launch_pdl(k_act8_forward<E, decltype(act)::value, decltype(gated)::value, R, true>, ctas, kThreads, 0, stream, a);
                    });
                });
            });
        });
    } else {
        const int64_t want = ((int64_t)a.all_groups + kThreads / 4 - 1) / (kThreads / 4);
        const int ctas = (int)(want < (int64_t)sm_count * kAct8Ctas ? want : (int64_t)sm_count * kAct8Ctas);
        e = with_dtype(p.dtype, [&](auto elem) {
            return with_bool(p.up != nullptr, [&](auto gated) {
                return with_act(p.act, [&](auto act) {
                    return launch_pdl(k_act8_forward_any<decltype(elem), decltype(act)::value, decltype(gated)::value>, ctas, kThreads, 0, stream, a);
                });
            });
        });
    }
    launch_end(stream);
    return e;
}

}  // namespace ogq

// Weight and bias gradient of a linear layer from its input kept in 8 bits: dW = dy^T x^, db = sum of dy's rows.
//   dW[o][i] = sum_t dy[t][o] x^[t][i]:  a product whose summed index t is the row of both operands.  x^ = code * 2^e is a bf16
// number, so nothing is lost by multiplying in bf16: dy in bf16 goes to the tensor cores as it is, dy in fp16 and fp32 as the sum
// of two and three bf16 terms (8 + 3 and 8 + 8 + 8 bits, exact down to 2^-133), stacked along t.
//   A pair of CTAs works on a tile of 256 x BN weights, 128 rows of t at a time: TMA brings dy's tile (swizzled, the operand as it lies
// in memory) and the codes; eight warps turn the codes into bf16 in shared memory (5 instructions for two values); one thread issues
// the MMAs of both CTAs.  Pairs: each SM holds half of x^'s tile, so every code is converted once for 256 columns of dy, and both
// operands cost half the shared memory traffic of single CTAs.
//   The tensor cores cut, not round, what they add to a running sum, which drifts by 2^-24 a step: a sum over 16,384 rows came out
// 9e-6 off, one over 1,024 rows 1e-6.  So a running sum is taken out of TMEM after 512 rows and added in registers, rounded to
// nearest, while the next one grows in the other half of TMEM.
//   Work is split by tile as long as there are tiles for all pairs; what is left (all of it, when weights are few and rows many) by
// steps of 128 rows, partial tiles joined by a second kernel in a fixed order.
//   What bounds it (16,384 x 4096 x 4096: this kernel alone in a short run 430 us, 1.28 PFLOP/s, the MMAs alone 281; the call with bias
// and join 510, and 545 to 560 in steady use, where power takes the clocks down): shared memory, which 64 rows of a tile keep busy for 640
// cycles (TMA writes 192, the converters read 64 and write 128, the MMAs read 256) where the MMAs take 512; in long runs, power.
#include <cuda.h>

#include "ogq_act8.cuh"
#include "ogq_internal.h"
#include "ogq_tcgen05.cuh"

namespace ogq {

// Rows of t per stage: fewer barriers and commits a row than with 64 (16,384 x 4096 x 4096, the product
// alone in a short run: 480 us, with 128 rows 437).
constexpr int kStepRows = 128;
constexpr int kFlush = 4;                      // steps per running sum
constexpr int kOperands = 2;                   // converted tiles of x^: one being written, one being multiplied
constexpr int kTileM = 256;                    // columns of dy per tile (both CTAs)
constexpr int kABytes = 128 * kStepRows * 2;   // dy's tile of one CTA
constexpr int kScaleBytes = kStepRows * 16;    // scales around those of a tile's (at most four) groups: 16 bytes a row by TMA, or two words
constexpr int kWgThreads = 640;                // a warpgroup for TMA, MMA, TMEM, scales and bias; two of converters; two that take sums out of TMEM
// Registers a thread of the three kinds; the block starts with 640 * 96 = 61,440, which the split must not exceed.
constexpr int kRegsStart = 96, kRegsControl = 64, kRegsConvert = 56, kRegsSums = 152;
static_assert(128 * kRegsControl + 256 * kRegsConvert + 256 * kRegsSums <= kWgThreads * kRegsStart, "a warpgroup would wait for registers for ever");
constexpr uint32_t kTmemColumns = 512;
constexpr int kMinSteps = 4;                   // of a part of a tile, and
constexpr int kMinSaved = 6;                   // steps that splitting has to save each pair: joining the parts takes 5 us, a step 0.9

template <int BN> struct WgShape {
    static constexpr int kCols = BN / 2;                          // columns of x^ that one CTA converts
    static constexpr int kOcts = kCols / 8;                       // a converter thread has eight of them, in
    static constexpr int kRowsAtOnce = 128 / kOcts;               // rows row, row + kRowsAtOnce, ...
    static constexpr int kRowsEach = kStepRows / 2 / kRowsAtOnce;  // of its warpgroup's half of the step
    static constexpr int kBBytes = kCols * kStepRows * 2;
    static constexpr int kRawBytes = kCols * kStepRows;
    static constexpr int kStages = BN == 256 ? 3 : 4;             // as many as fit: loads under way
    static constexpr int kRing = kStages * (kABytes + kRawBytes + kScaleBytes) + kOperands * kBBytes;
    static constexpr int kSmem = kRing + 8 * 32 * 9 * 4 + 1024;    // + patches of rows on their way out, + alignment to the swizzle's 1024 bytes
    static_assert(kABytes % 1024 == 0 && kBBytes % 1024 == 0, "the swizzle goes by the address");
    static_assert(kSmem <= 226 * 1024, "shared memory");
    static constexpr int kSlotFloats = 128 * BN;                  // a partial tile of one CTA
};

__host__ __device__ inline int64_t bias_pitch(int64_t out_cols) { return (out_cols + 3) / 4 * 4; }

struct WgArgs {
    const uint8_t* scales;
    float* dw;
    float* slots;
    int64_t cols, out_cols;
    int64_t rows;       // of this launch
    int groups;         // of a row
    int tiles_m, tiles_n;
    int steps;          // of a tile: terms * steps_x
    int steps_x;        // steps over x^'s rows
    int last_rows;      // of the last of them that are multiplied, a multiple of 16 (dy's tile is zero below, x^ is not converted)
    int pairs;
    int whole;          // tiles per pair that are done alone
    int64_t rest;       // steps of the tiles left
    int64_t per;        // of them per pair
    bool accumulate;
    bool wide;          // 32-byte stores
    bool tma_scales;    // a multiple of 16 groups: TMA copies the scales
    // Bias (db not null): from partial sums over `chunks` parts of the rows, or (chunks = 0, one step) from dy.
    float* db;
    const float* bias_parts;  // [chunks][bias_pitch]
    int chunks;
    const uint16_t* dy;       // as TMA reads it: bf16, dy_rows rows of stride ld_dy
    int64_t ld_dy, dy_rows;
};

// The pieces of work of one pair: (tile, steps [k0, k1)), the same sequence in every role.
struct WgWork {
    int i;
    int64_t at, end;
    int tile, k0, k1, slot;  // slot < 0: the whole sum
    __device__ __forceinline__ WgWork(const WgArgs& a, int pair) : i(0), tile(0), k0(0), k1(0), slot(-1)
    {
        at = (int64_t)pair * a.per;
        if (at > a.rest) at = a.rest;
        end = at + a.per < a.rest ? at + a.per : a.rest;
        first_ = true;
    }
    __device__ __forceinline__ bool next(const WgArgs& a, int pair)
    {
        if (i < a.whole) {
            tile = pair + i * a.pairs;
            k0 = 0;
            k1 = a.steps;
            ++i;
            return true;
        }
        if (at >= end) return false;
        const int j = (int)(at / a.steps);
        tile = a.whole * a.pairs + j;
        k0 = (int)(at - (int64_t)j * a.steps);
        const int64_t left = end - at;
        k1 = (int)(k0 + left < a.steps ? k0 + left : a.steps);
        slot = k0 == 0 && k1 == a.steps ? -1 : first_ ? 0 : 1;
        first_ = false;
        at += k1 - k0;
        return true;
    }
    bool first_;
};

// Tiles in columns of eight: those that run side by side read few different rows of both operands.
__device__ __forceinline__ void wg_tile_place(int tile, int tiles_m, int tiles_n, int& m, int& n)
{
    const int band = tile / (8 * tiles_n), in = tile - band * 8 * tiles_n;
    const int height = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
    n = in / height;
    m = band * 8 + in - n * height;
}

// Two codes of a word, already spread to the low bytes of its halves, times the unit: 128 + (low seven bits) less 128, or 256
// where the sign is set, both bf16 numbers whose bits are an OR away.
__device__ __forceinline__ uint32_t wg_value2(uint32_t p, __nv_bfloat162 unit)
{
    const uint32_t a = (p & 0x007f007fu) | 0x43004300u, b = (p & 0x00800080u) | 0x43004300u;
    const __nv_bfloat162 q = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    const __nv_bfloat162 v = __hmul2(q, unit);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight codes of row t and their scale byte into the row's place in the operand.
__device__ __forceinline__ void wg_put8(uint32_t x, uint32_t y, uint32_t byte, uint32_t b, int t, int oct)
{
    const uint32_t both = byte * 0x800080u;  // the byte is a bf16 number's exponent
    const __nv_bfloat162 unit = *reinterpret_cast<const __nv_bfloat162*>(&both);
    const uint32_t v0 = wg_value2(__byte_perm(x, 0, 0x4140), unit), v1 = wg_value2(__byte_perm(x, 0, 0x4342), unit);
    const uint32_t v2 = wg_value2(__byte_perm(y, 0, 0x4140), unit), v3 = wg_value2(__byte_perm(y, 0, 0x4342), unit);
    const uint32_t at = b + (oct >> 3) * (kStepRows * 128) + t * 128 + (((oct ^ t) & 7) << 4);
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(v0), "r"(v1), "r"(v2), "r"(v3) : "memory");
}

// This thread's rows below `rows`, eight codes each, of the stage's codes, scales (from this thread's byte on) and place for the
// operand.  Eight lanes write the 128 bytes of a row of a swizzled block: no bank conflicts.
template <int BN>
__device__ __forceinline__ void wg_convert(uint32_t raw, uint32_t scales, int pitch, uint32_t b, int row, int oct, int rows)
{
    constexpr int kCols = WgShape<BN>::kCols, kEach = WgShape<BN>::kRowsEach, kStep = WgShape<BN>::kRowsAtOnce;
    if (rows < kStepRows) {  // the last step
#pragma unroll 1
        for (int t = row; t < rows && t < row + kEach * kStep; t += kStep) {
            uint32_t x, y, u;
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(raw + t * kCols + oct * 8));
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(u) : "r"(scales + t * pitch));
            wg_put8(x, y, u, b, t, oct);
        }
        return;
    }
    uint32_t c[kEach][2], u[kEach];  // all loads before the first store, which none could pass
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int t = row + kStep * j;
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(c[j][0]), "=r"(c[j][1]) : "r"(raw + t * kCols + oct * 8));
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(u[j]) : "r"(scales + t * pitch));
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) wg_put8(c[j][0], c[j][1], u[j], b, row + kStep * j, oct);
}

__device__ __forceinline__ void store8_wide(float* p, const float* v)
{
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}

// Eight neighbouring weights of row o from column i on; cols is a multiple of 8 and rows begin on 32-byte boundaries.
__device__ __forceinline__ void wg_store8(const WgArgs& a, int64_t o, int64_t i, float (&v)[8])
{
    if (o >= a.out_cols || i >= a.cols) return;
    float* w = a.dw + o * a.cols + i;
    if (a.accumulate) {
        const float4 p = *reinterpret_cast<const float4*>(w), q = *reinterpret_cast<const float4*>(w + 4);
        v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        v[4] += q.x; v[5] += q.y; v[6] += q.z; v[7] += q.w;
    }
    store8_wide(w, v);
}

// The same for any cols and address, by a warp: lane l has row o + l.  Through shared memory, so that eight lanes write a row's eight
// weights (300 x 999 x 2001: 35 -> 21 us).
constexpr int kPatch = 32 * 9;  // floats of a warp
__device__ __forceinline__ void wg_store_patch(const WgArgs& a, float* patch, int64_t o, int64_t i, const float* v, int lane)
{
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) patch[lane * 9 + j] = v[j];
    __syncwarp();
    const int64_t c = i + (lane & 7);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t r = o + k * 4 + (lane >> 3);
        if (r >= a.out_cols || c >= a.cols) continue;
        float* w = a.dw + r * a.cols + c;
        const float x = patch[(k * 4 + (lane >> 3)) * 9 + (lane & 7)];
        *w = a.accumulate ? *w + x : x;
    }
}

// Four lanes with four eights of values each: lane j's eight r becomes lane r's eight j.
__device__ __forceinline__ void wg_exchange(float* v, int lane)
{
#pragma unroll
    for (int bit = 1; bit <= 2; bit *= 2) {
        const bool high = lane & bit;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (r & bit) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float& a = v[r * 8 + j];
                float& b = v[(r | bit) * 8 + j];
                const float got = __shfl_xor_sync(0xffffffffu, high ? a : b, bit);
                if (high) a = got;
                else b = got;
            }
        }
    }
}

// db of four columns from o on, a multiple of 4.
__device__ __forceinline__ void wg_bias(const WgArgs& a, int64_t o)
{
    if (o >= a.out_cols) return;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.chunks > 0) {
#pragma unroll 4
        for (int k = 0; k < a.chunks; ++k) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(a.bias_parts + k * bias_pitch(a.out_cols) + o));
            sum[0] = __fadd_rn(sum[0], v.x);
            sum[1] = __fadd_rn(sum[1], v.y);
            sum[2] = __fadd_rn(sum[2], v.z);
            sum[3] = __fadd_rn(sum[3], v.w);
        }
    } else {
        const uint16_t* p = a.dy + o;
        const int rows = (int)a.dy_rows;
        constexpr int kAtOnce = 8;
        for (int t = 0; t < rows; t += kAtOnce) {
            uint2 v[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) v[k] = make_uint2(0u, 0u);
            if (o + 3 < a.out_cols) {
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
                    if (t + k < rows) v[k] = *reinterpret_cast<const uint2*>(p + (t + k) * a.ld_dy);
            } else {
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (t + k >= rows) break;
                    const uint16_t* q = p + (t + k) * a.ld_dy;
                    v[k].x = q[0];
                    if (o + 1 < a.out_cols) v[k].x |= (uint32_t)q[1] << 16;
                    if (o + 2 < a.out_cols) v[k].y = q[2];
                }
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                sum[0] = __fadd_rn(sum[0], __uint_as_float(v[k].x << 16));
                sum[1] = __fadd_rn(sum[1], __uint_as_float(v[k].x & 0xffff0000u));
                sum[2] = __fadd_rn(sum[2], __uint_as_float(v[k].y << 16));
                sum[3] = __fadd_rn(sum[3], __uint_as_float(v[k].y & 0xffff0000u));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (o + j < a.out_cols) a.db[o + j] = a.accumulate ? a.db[o + j] + sum[j] : sum[j];
}

// WIDE: rows of dW are whole 32-byte pieces
template <int BN, bool WIDE>
__global__ void __launch_bounds__(kWgThreads, 1) __cluster_dims__(2, 1, 1)
k_wgrad(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_x,
        const __grid_constant__ CUtensorMap map_scales, const __grid_constant__ WgArgs a)
{
    using S = WgShape<BN>;
    extern __shared__ uint8_t smem_raw[];
    constexpr int kStages = S::kStages;
    __shared__ uint64_t bars[4 * kStages + kOperands + 4];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = (int)(blockIdx.x >> 1);
    const uint32_t bar0 = smem_u32(bars);
    // dy_here (leader's): both CTAs' tiles of dy are here.  raw_here: codes and scales are here; raw_free: they are converted.
    // op_here (leader's): both CTAs' converted tiles are.  done (both): the step is multiplied, its tile of dy and its converted
    // tile are free (one barrier for both: a commit holds the issuing thread up for 150 cycles and more).
    // sum (both): a running sum is complete; taken (leader's): both CTAs have read it.
    const auto dy_here = [&](int s) { return bar0 + 8u * s; };
    const auto done = [&](int s) { return bar0 + 8u * (kStages + s); };
    const auto raw_here = [&](int s) { return bar0 + 8u * (2 * kStages + s); };
    const auto raw_free = [&](int s) { return bar0 + 8u * (3 * kStages + s); };
    const auto op_here = [&](int b) { return bar0 + 8u * (4 * kStages + b); };
    const auto sum = [&](int d) { return bar0 + 8u * (4 * kStages + kOperands + d); };
    const auto taken = [&](int d) { return bar0 + 8u * (4 * kStages + kOperands + 2 + d); };
    const auto stage_a = [&](int s) { return base + s * kABytes; };
    const auto operand_b = [&](int b) { return base + kStages * kABytes + b * S::kBBytes; };
    const auto stage_raw = [&](int s) { return base + kStages * kABytes + kOperands * S::kBBytes + s * S::kRawBytes; };
    const auto stage_scales = [&](int s) { return base + kStages * (kABytes + S::kRawBytes) + kOperands * S::kBBytes + s * kScaleBytes; };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(dy_here(s), 1);
            mbar_init(done(s), 1);
            mbar_init(raw_here(s), a.tma_scales ? 1 : 33);  // TMA's, and those of the lanes that copy the scales
            mbar_init(raw_free(s), 8);
        }
        for (int b = 0; b < kOperands; ++b) mbar_init(op_here(b), 16);
        for (int d = 0; d < 2; ++d) {
            mbar_init(sum(d), 1);
            mbar_init(taken(d), 16);
        }
        failed = 0;
        mbar_init_fence();
        tma_prefetch_map(&map_dy);
        tma_prefetch_map(&map_x);
    }
    if (warp == 2) tmem_alloc_pair(smem_u32(&tmem_base), kTmemColumns);
    tcgen05_fence_before();
    cluster_sync();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    pdl_wait();
    pdl_launch_dependents();

    if (warp < 4) {
        fewer_registers<kRegsControl>();
        if (warp == 0 && lane == 0) {  // dy, by TMA
            WgWork w(a, pair);
            int s = 0;
            uint32_t phase = 1;  // the first pass over the stages finds them free
            bool ok = true;
            const uint32_t here = map_to(dy_here(0), 0);
            while (ok && w.next(a, pair)) {
                int m, n;
                wg_tile_place(w.tile, a.tiles_m, a.tiles_n, m, n);
                const int o = m * kTileM + (int)rank * 128;
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = mbar_wait(done(s), phase, &failed))) break;
                    if (rank == 0) mbar_expect(dy_here(s), 2 * kABytes);
                    tma_load_pair(stage_a(s), &map_dy, o, k * kStepRows, here + 8 * s);
                    tma_load_pair(stage_a(s) + kABytes / 2, &map_dy, o + 64, k * kStepRows, here + 8 * s);
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
            }
            // Until the last copies have landed: a stage is free again when its MMAs, and so its copies, are done.
            for (int k = 0; k < kStages; ++k) {
                if (!mbar_wait(done(s), phase, &failed)) break;
                if (++s == kStages) { s = 0; phase ^= 1; }
            }
        } else if (warp == 2 && lane == 0) {  // codes, by TMA (a thread for both kinds took 750 cycles a step to issue them)
            WgWork w(a, pair);
            int s = 0;
            uint32_t phase = 1;
            bool ok = true;
            while (ok && w.next(a, pair)) {
                int m, n;
                wg_tile_place(w.tile, a.tiles_m, a.tiles_n, m, n);
                const int i = n * BN + (int)rank * S::kCols;
                int x = w.k0 % a.steps_x;
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = mbar_wait(raw_free(s), phase, &failed))) break;
                    mbar_expect(raw_here(s), S::kRawBytes + (a.tma_scales ? kScaleBytes : 0));
                    tma_load_pair(stage_raw(s), &map_x, i, x * kStepRows, raw_here(s));
                    if (a.tma_scales) tma_load_pair(stage_scales(s), &map_scales, i / kAct8Group & ~15, x * kStepRows, raw_here(s));
                    if (++x == a.steps_x) x = 0;
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
            }
        } else if (warp == 1 && lane == 0 && rank == 0) {  // MMA of both CTAs
            WgWork w(a, pair);
            int s = 0, b = 0, d = 0;
            uint32_t phase = 0, bphase = 0, dphase = 1;
            bool ok = true;
            constexpr uint32_t instruction = instruction_bf16(kTileM, BN);
            while (ok && w.next(a, pair)) {
                int x = w.k0 % a.steps_x;
                for (int k = w.k0; ok && k < w.k1; k += kFlush) {
                    const int last = k + kFlush < w.k1 ? k + kFlush : w.k1;
                    if (!(ok = mbar_wait(taken(d), dphase, &failed))) break;
                    tcgen05_fence_after();
                    for (int q = k; q < last; ++q) {
                        if (!(ok = mbar_wait(dy_here(s), phase, &failed) && mbar_wait(op_here(b), bphase, &failed))) break;
                        tcgen05_fence_after();
                        const uint64_t da = tile_descriptor(stage_a(s), kStepRows * 128), db = tile_descriptor(operand_b(b), kStepRows * 128);
                        if (++x < a.steps_x) {
#pragma unroll
                            for (int j = 0; j < kStepRows / 16; ++j)  // 16 rows are 2048 bytes on
                                mma_bf16_pair(tmem + d * BN, da + j * (2048 >> 4), db + j * (2048 >> 4), instruction, q > k || j > 0);
                        } else {
                            x = 0;
                            for (int j = 0; j < a.last_rows / 16; ++j)
                                mma_bf16_pair(tmem + d * BN, da + j * (2048 >> 4), db + j * (2048 >> 4), instruction, q > k || j > 0);
                        }
                        mma_commit_pair(done(s));
                        if (++b == kOperands) { b = 0; bphase ^= 1; }
                        if (++s == kStages) { s = 0; phase ^= 1; }
                    }
                    if (!ok) break;
                    mma_commit_pair(sum(d));
                    if (++d == 2) { d = 0; dphase ^= 1; }
                }
            }
        }
        else if (warp == 3) {
            if (a.db) {  // bias: of each column of tiles, by the CTAs that begin its first tile
                WgWork w(a, pair);
                while (w.next(a, pair)) {
                    int m, n;
                    wg_tile_place(w.tile, a.tiles_m, a.tiles_n, m, n);
                    if (n == 0 && w.k0 == 0) wg_bias(a, (int64_t)m * kTileM + rank * 128 + lane * 4);
                }
            }
            // scales that TMA does not copy: the aligned words around each row's bytes, never past the end
            WgWork w(a, pair);
            int s = 0;
            uint32_t phase = 1;
            bool ok = true;
            const int64_t all = a.rows * a.groups;
            while (!a.tma_scales && ok && w.next(a, pair)) {
                int m, n;
                wg_tile_place(w.tile, a.tiles_m, a.tiles_n, m, n);
                const int first = (n * BN + (int)rank * S::kCols) / kAct8Group;
                int x = w.k0 % a.steps_x;
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(raw_free(s), phase, &failed)))) break;
#pragma unroll
                    for (int r = 0; r < kStepRows / 16; ++r) {
                        const int row = lane + (r >> 1) * 32;
                        const int64_t t = (int64_t)x * kStepRows + row;
                        const int64_t at = ((t * a.groups + first) & ~(int64_t)3) + (r & 1) * 4;
                        const int64_t left = t < a.rows ? all - at : 0;
                        copy4_async(stage_scales(s) + row * 8 + (r & 1) * 4, a.scales + (left > 0 ? at : 0), left >= 4 ? 4 : left > 0 ? (int)left : 0);
                    }
                    copies_arrive(raw_here(s));
                    if (++x == a.steps_x) x = 0;
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
            }
        }
    } else if (warp < 12) {  // converters: each warpgroup half of the rows
        fewer_registers<kRegsConvert>();
        const int id = threadIdx.x & 127;
        const int oct = id % S::kOcts, row = ((warp - 4) >> 2) * (kStepRows / 2) + id / S::kOcts;
        WgWork w(a, pair);
        // the operand's place is free when the step kOperands before this one is done (none for the first kOperands)
        int s = 0, b = 0, before = kStages - kOperands;
        uint32_t phase = 0, before_phase = 1;
        bool ok = true;
        while (ok && w.next(a, pair)) {
            int m, n;
            wg_tile_place(w.tile, a.tiles_m, a.tiles_n, m, n);
            // this thread's byte of a row's; of words, the first holds the row's at a place that is the same eight rows on
            const int first = (n * BN + (int)rank * S::kCols) / kAct8Group;
            const int byte = (a.tma_scales ? first & 15 : (row * a.groups + first) & 3) + oct / 4;
            int x = w.k0 % a.steps_x;
            for (int k = w.k0; k < w.k1; ++k) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(raw_here(s), phase, &failed) && mbar_wait(done(before), before_phase, &failed)))) break;
                wg_convert<BN>(stage_raw(s), stage_scales(s) + byte, a.tma_scales ? 16 : 8, operand_b(b), row, oct, x + 1 == a.steps_x ? a.last_rows : kStepRows);
                if (++x == a.steps_x) x = 0;
                fence_async_shared();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_cluster(map_to(op_here(b), 0));
                    mbar_arrive(raw_free(s));
                }
                if (++s == kStages) { s = 0; phase ^= 1; }
                if (++before == kStages) { before = 0; before_phase ^= 1; }
                if (++b == kOperands) b = 0;
            }
        }
    } else {  // sums out of TMEM, and out
        more_registers<kRegsSums>();
        constexpr int kHalf = BN / 2;
        const int quarter = warp & 3, half = (warp - 12) >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        WgWork w(a, pair);
        int d = 0;
        uint32_t dphase = 0;
        bool ok = true;
        while (ok && w.next(a, pair)) {
            float acc[kHalf];
#pragma unroll
            for (int j = 0; j < kHalf; ++j) acc[j] = 0.f;
            for (int k = w.k0; k < w.k1; k += kFlush) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(sum(d), dphase, &failed)))) break;
                tcgen05_fence_after();
#pragma unroll
                for (int c = 0; c < kHalf; c += 16) {
                    float v[16];
                    tmem_load16(tmem + lanes + d * BN + half * kHalf + c, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) acc[c + j] = __fadd_rn(acc[c + j], v[j]);
                }
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to(taken(d), 0));
                if (++d == 2) { d = 0; dphase ^= 1; }
            }
            if (!ok) {
#pragma unroll
                for (int j = 0; j < kHalf; ++j) acc[j] = __uint_as_float(0x7fc00000u);  // a wait that ran out is not to be missed
            }
            int m, n;
            wg_tile_place(w.tile, a.tiles_m, a.tiles_n, m, n);
            const int row = quarter * 32 + lane;
            if (w.slot < 0) {
                if constexpr (!WIDE) {
                    float* patch = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)) + S::kRing) + (warp - 12) * kPatch;
                    const int64_t o = (int64_t)m * kTileM + rank * 128 + quarter * 32, i = (int64_t)n * BN + half * kHalf;
#pragma unroll
                    for (int c = 0; c < kHalf; c += 8)
                        if (i + c < a.cols) wg_store_patch(a, patch, o, i + c, acc + c, lane);
                } else {
                    // Four lanes exchange their rows' eights of columns, so that they write 128 bytes of one row at a time (a row a lane, 32
                    // bytes at a time: 4.1 us for a tile).
                    const int64_t o = (int64_t)m * kTileM + rank * 128 + (row & ~3), i = (int64_t)n * BN + half * kHalf + (lane & 3) * 8;
#pragma unroll
                    for (int c = 0; c < kHalf; c += 32) {
                        wg_exchange(acc + c, lane);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float v[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[j] = acc[c + r * 8 + j];
                            wg_store8(a, o + r, i + c, v);
                        }
                    }
                }
            } else {
                float* slot = a.slots + ((int64_t)(pair * 2 + w.slot) * 2 + rank) * S::kSlotFloats;
#pragma unroll
                for (int c = 0; c < kHalf; c += 8)
                    if ((int64_t)n * BN + half * kHalf + c < a.cols) store8_wide(slot + ((half * kHalf + c) / 8 * 128 + row) * 8, acc + c);
            }
        }
    }
    __syncwarp();
    tcgen05_fence_before();
    cluster_sync();
    tcgen05_fence_after();
    if (warp == 2) tmem_free_pair(tmem, kTmemColumns);
}

// Joins the partial tiles: eight weights a thread; PARTS > 1: many pairs' parts of few tiles, each PARTS-th summed by another
// warp of the CTA, then in order.  A CTA takes 256 / PARTS rows of eight columns.
template <int BN, int PARTS>
__global__ void __launch_bounds__(kThreads) k_wgrad_join(const __grid_constant__ WgArgs a)
{
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kRows = kThreads / PARTS;  // of the tile's 256 x BN/8 pieces (CTA-of-the-pair, octet, row)
    __shared__ float4 sh[PARTS > 1 ? PARTS : 1][PARTS > 1 ? kRows : 1][2];
    __shared__ float patches[kRows / 32][kPatch];
    constexpr int kPerTile = 256 * (BN / 8) / kRows;
    const int j = blockIdx.x / kPerTile;
    const int part = threadIdx.x / kRows, r = threadIdx.x - part * kRows;
    const int piece = (blockIdx.x - j * kPerTile) * kRows + r;
    const int rank = piece / (128 * (BN / 8)), in = piece - rank * (128 * (BN / 8));
    const int oct = in / 128, row = in - oct * 128;
    int m, n;
    wg_tile_place(a.whole * a.pairs + j, a.tiles_m, a.tiles_n, m, n);
    const int64_t begin = (int64_t)j * a.steps, first = begin / a.per, last = (begin + a.steps - 1) / a.per;
    if (first == last) return;  // done by one pair
    if ((int64_t)n * BN + oct * 8 >= a.cols) return;  // all of the CTA: its rows have the same eight columns
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    constexpr int kAtOnce = 4;
    for (int64_t p0 = first + part; p0 <= last; p0 += PARTS * kAtOnce) {
        float4 x[kAtOnce], y[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t p = p0 + k * PARTS;
            x[k] = y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (p <= last) {
                const int slot = p * a.per < begin ? 1 : 0;  // a pair that begins before this tile has it second
                const float4* s = reinterpret_cast<const float4*>(a.slots + ((p * 2 + slot) * 2 + rank) * WgShape<BN>::kSlotFloats + (int64_t)in * 8);
                x[k] = __ldcg(s);
                y[k] = __ldcg(s + 1);
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            v[0] += x[k].x; v[1] += x[k].y; v[2] += x[k].z; v[3] += x[k].w;
            v[4] += y[k].x; v[5] += y[k].y; v[6] += y[k].z; v[7] += y[k].w;
        }
    }
    if constexpr (PARTS > 1) {
        sh[part][r][0] = make_float4(v[0], v[1], v[2], v[3]);
        sh[part][r][1] = make_float4(v[4], v[5], v[6], v[7]);
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int q = 1; q < PARTS; ++q) {
            const float4 x = sh[q][r][0], y = sh[q][r][1];
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
    }
    const int64_t o = (int64_t)m * kTileM + rank * 128 + row, i = (int64_t)n * BN + oct * 8;
    if (a.wide) wg_store8(a, o, i, v);
    else wg_store_patch(a, patches[r / 32], o - r % 32, i, v, r % 32);  // (a warp has 32 rows in a row)
}

// ---------------------------------------------------------------------------
// Operands that TMA cannot read as they are (fp16, fp32, rows off 16-byte boundaries) are laid out in the scratch first:
// dy as bf16 terms stacked along t, each of `padded` rows (a multiple of a step's, zeros behind the last), and the codes with rows of
// a multiple of 16 bytes; scales off 4-byte boundaries are copied too.
// ---------------------------------------------------------------------------
struct WgLayout {
    const void* dy; int64_t ld_dy;
    const int8_t* codes;
    uint16_t* terms; int64_t ld_terms;   // null: dy is read as it is
    int8_t* kept; int64_t ld_kept;       // null: the codes are
    const uint8_t* scales; uint8_t* scales_to; int64_t n_scales;  // scales_to null: the scales are
    int64_t rows, padded, cols, out_cols;
};

// Cut, not rounded, so that the largest fp32 numbers do not become infinite; what is left is exact.  Infinities and NaN have a
// first term only.
template <int TERMS>
__device__ __forceinline__ void wg_split(float v, uint16_t (&t)[TERMS])
{
    const bool finite = (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
        uint32_t b = __float_as_uint(v);
        if (k == 0 && !finite && (b & 0x007fffffu)) b |= 0x00400000u;  // a NaN stays one when cut
        t[k] = (uint16_t)(k > 0 && !finite ? 0u : b >> 16);
        v = __fsub_rn(v, __uint_as_float(b & 0xffff0000u));
    }
}

template <class E, int TERMS>
__global__ void __launch_bounds__(kThreads) k_wgrad_layout(const __grid_constant__ WgLayout a)
{
    pdl_wait();
    pdl_launch_dependents();
    const int64_t stride = (int64_t)gridDim.x * kThreads, id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (a.terms) {
        const int64_t octs = a.ld_terms / 8, n = a.padded * octs;
        for (int64_t i = id; i < n; i += stride) {
            const int64_t t = i / octs, c = (i - t * octs) * 8;
            uint16_t v[8][TERMS];
#pragma unroll
            for (int j = 0; j < 8; ++j) wg_split<TERMS>(t < a.rows && c + j < a.out_cols ? load1((const E*)a.dy + t * a.ld_dy + c + j) : 0.f, v[j]);
#pragma unroll
            for (int k = 0; k < TERMS; ++k)
                *reinterpret_cast<uint4*>(a.terms + (k * a.padded + t) * a.ld_terms + c) =
                    make_uint4(v[0][k] | (uint32_t)v[1][k] << 16, v[2][k] | (uint32_t)v[3][k] << 16, v[4][k] | (uint32_t)v[5][k] << 16,
                               v[6][k] | (uint32_t)v[7][k] << 16);
        }
    }
    if (a.kept) {
        const int64_t pieces = a.ld_kept / 16, n = a.rows * pieces;
        for (int64_t i = id; i < n; i += stride) {
            const int64_t t = i / pieces, c = (i - t * pieces) * 16;
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < a.cols) w[j / 4] |= (uint32_t)(uint8_t)a.codes[t * a.cols + c + j] << (j % 4 * 8);
            *reinterpret_cast<uint4*>(a.kept + t * a.ld_kept + c) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    if (a.scales_to)
        for (int64_t i = id; i < a.n_scales; i += stride) a.scales_to[i] = a.scales[i];
}

// ---------------------------------------------------------------------------
// Bias: a CTA sums V columns a lane over its rows; several chunks of rows leave partial sums for the second kernel.
// ---------------------------------------------------------------------------
struct WgBias {
    const void* dy; int64_t ld_dy;
    int64_t rows, out_cols, chunk;
    float* part; float* db;
    int chunks, ctiles;
    bool accumulate;
};

template <class E, int V>
__global__ void __launch_bounds__(kThreads) k_wgrad_bias(const __grid_constant__ WgBias a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float sh[kWarps][32 * V];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t k = blockIdx.x / a.ctiles, c = ((blockIdx.x - k * a.ctiles) * 32 + lane) * V;
    const int64_t end = (k + 1) * a.chunk < a.rows ? (k + 1) * a.chunk : a.rows;
    float s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 0.f;
    if (c < a.out_cols) {
        constexpr int kAtOnce = 8;
        const E* p = (const E*)a.dy + c;
        for (int64_t t = k * a.chunk + warp; t < end; t += kAtOnce * kWarps) {
            if constexpr (V == 8) {
                Raw8<E> r[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) r[u] = t + u * kWarps < end ? load_raw8(p + (t + u * kWarps) * a.ld_dy) : zero_raw8<E>();
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    float v[V];
                    unpack8(r[u], v);
#pragma unroll
                    for (int j = 0; j < V; ++j) s[j] = __fadd_rn(s[j], v[j]);
                }
            } else {
                float v[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) v[u] = t + u * kWarps < end ? load1(p + (t + u * kWarps) * a.ld_dy) : 0.f;
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) s[0] = __fadd_rn(s[0], v[u]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sh[warp][lane * V + j] = s[j];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * V; i += kThreads) {
        const int64_t o = (blockIdx.x - k * a.ctiles) * 32 * V + i;
        if (o >= a.out_cols) break;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum += sh[w][i];
        if (a.chunks == 1) a.db[o] = a.accumulate ? a.db[o] + sum : sum;
        else a.part[k * bias_pitch(a.out_cols) + o] = sum;
    }
}

// Many chunks: a CTA joins 32 columns, eight chunks at a time.
__global__ void __launch_bounds__(kThreads) k_wgrad_bias_join(const __grid_constant__ WgBias a)
{
    pdl_wait();
    pdl_launch_dependents();
    __shared__ float sh[kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t o = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (o < a.out_cols) {
#pragma unroll 8
        for (int k = warp; k < a.chunks; k += kWarps) s = __fadd_rn(s, __ldcg(a.part + k * bias_pitch(a.out_cols) + o));
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp || o >= a.out_cols) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s = __fadd_rn(s, sh[w][lane]);
    a.db[o] = a.accumulate ? a.db[o] + s : s;
}

// All sums empty.
__global__ void __launch_bounds__(kThreads) k_wgrad_zero(float* p, int64_t n, float* q, int64_t m)
{
    pdl_wait();
    pdl_launch_dependents();
    const int64_t stride = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n + m; i += stride) {
        if (i < n) p[i] = 0.f;
        else q[i - n] = 0.f;
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
namespace {

constexpr int64_t kLayoutBytes = (int64_t)40 << 20;  // of operands laid out at a time: they stay in L2 until they are read
constexpr int kBiasCtas = 4;                         // per SM
constexpr int kBiasParts = 40;                       // up to these are joined by the product's kernel
constexpr int64_t kBiasRows = 64;                    // up to these, no kernel of its own

int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
int terms_of(int dtype) { return dtype == OGQ_F32 ? 3 : dtype == OGQ_F16 ? 2 : 1; }

struct Plan {
    bool lay_dy, lay_x, lay_s;
    int terms, pairs;
    int64_t ld_terms, ld_kept, rows;  // rows per launch
    int64_t slots_bytes, bias_bytes, terms_bytes, kept_bytes, scales_bytes;
    int64_t bias_chunk;
    int bias_chunks;
};

Plan make_plan(int64_t rows, int64_t cols, int64_t out_cols, int dtype, bool lay_dy, bool lay_x, bool lay_s, int sm_count)
{
    Plan p = {};
    p.lay_dy = lay_dy;
    p.lay_x = lay_x;
    p.lay_s = lay_s;
    p.terms = terms_of(dtype);
    p.pairs = sm_count / 2;
    p.ld_terms = up_to(out_cols, 8);
    p.ld_kept = up_to(cols, 16);
    p.rows = rows;
    if (lay_dy || lay_x || lay_s) {
        const int64_t per_row = (lay_dy ? p.terms * p.ld_terms * 2 : 0) + (lay_x ? p.ld_kept : 0) + (lay_s ? act8_groups(cols) : 0);
        int64_t most = kLayoutBytes / (per_row > 0 ? per_row : 1) / kStepRows * kStepRows;
        if (most < 4 * kStepRows) most = 4 * kStepRows;
        if (p.rows > most) p.rows = most;
    }
    const int64_t padded = up_to(p.rows, kStepRows);
    p.terms_bytes = lay_dy ? up_to(p.terms * padded * p.ld_terms * 2, 256) : 0;
    p.kept_bytes = lay_x ? up_to(p.rows * p.ld_kept, 256) : 0;
    p.scales_bytes = lay_s ? up_to(p.rows * act8_groups(cols), 256) : 0;
    p.slots_bytes = (int64_t)p.pairs * 4 * WgShape<256>::kSlotFloats * 4;
    // chunks of rows for the bias: enough CTAs, each of 64 rows or more
    const int64_t ctiles = (out_cols + 255) / 256;
    int64_t chunks = (int64_t)sm_count * kBiasCtas / ctiles;
    if (chunks > (rows + 63) / 64) chunks = (rows + 63) / 64;
    if (chunks < 1) chunks = 1;
    p.bias_chunk = (rows + chunks - 1) / chunks;
    if (p.bias_chunk < 1) p.bias_chunk = 1;
    p.bias_chunks = (int)((rows + p.bias_chunk - 1) / p.bias_chunk);
    if (p.bias_chunks < 1) p.bias_chunks = 1;
    p.bias_bytes = up_to(p.bias_chunks * bias_pitch(out_cols) * 4, 256);
    return p;
}

// cuTensorMapEncodeTiled, looked up once per process.
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) p = nullptr;
        return (EncodeTiled)p;
    }();
    return f;
}

// A matrix of bf16 (swizzled boxes) or bytes.
bool make_map(CUtensorMap* map, const void* p, bool bf16, int64_t cols, int64_t rows, int64_t ld_bytes, int box_cols)
{
    const EncodeTiled f = encode_tiled();
    if (!f) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld_bytes};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)kStepRows}, steps[2] = {1, 1};
    return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, steps,
             CU_TENSOR_MAP_INTERLEAVE_NONE, bf16 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN>
cudaError_t launch_product(const CUtensorMap& map_dy, const CUtensorMap& map_x, const CUtensorMap& map_scales, WgArgs a, cudaStream_t stream)
{
    a.tiles_m = (int)((a.out_cols + kTileM - 1) / kTileM);
    a.tiles_n = (int)((a.cols + BN - 1) / BN);
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    if (tiles > 0x3fffffff) return cudaErrorInvalidValue;
    a.whole = (int)(tiles / a.pairs);
    const int64_t left = tiles - (int64_t)a.whole * a.pairs;
    a.rest = left * a.steps;
    a.per = (a.rest + a.pairs - 1) / a.pairs;
    if (a.per < kMinSteps) a.per = kMinSteps;
    if (left == 0 || a.per + kMinSaved > a.steps) a.per = a.steps;
    const int64_t busy = a.whole ? a.pairs : (a.rest + a.per - 1) / a.per;
    // A build whose kernel starts with fewer registers than the split needs would wait for them for ever: it is not launched.
    static const bool starts_with_all = [] {
        cudaFuncAttributes f, g;
        return cudaFuncGetAttributes(&f, k_wgrad<BN, false>) == cudaSuccess && f.numRegs >= kRegsStart &&
               cudaFuncGetAttributes(&g, k_wgrad<BN, true>) == cudaSuccess && g.numRegs >= kRegsStart;
    }();
    if (!starts_with_all) return cudaErrorInvalidConfiguration;
    const auto kernel = a.wide ? k_wgrad<BN, true> : k_wgrad<BN, false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, WgShape<BN>::kSmem);
    if (e != cudaSuccess) return e;
    launch_begin("k_wgrad", stream);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * busy));
    cfg.blockDim = dim3(kWgThreads);
    cfg.dynamicSmemBytes = WgShape<BN>::kSmem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, map_dy, map_x, map_scales, a);
    launch_end(stream);
    if (e != cudaSuccess || left == 0 || a.per % a.steps == 0) return e;  // no tile is split
    launch_begin("k_wgrad_join", stream);
    if (a.steps >= 8 * a.per)
        e = launch_pdl(k_wgrad_join<BN, 8>, (int)(left * 256 * (BN / 8) / 32), kThreads, 0, stream, a);
    else
        e = launch_pdl(k_wgrad_join<BN, 1>, (int)(left * 256 * (BN / 8) / 256), kThreads, 0, stream, a);
    launch_end(stream);
    return e;
}

}  // namespace

size_t ws_bytes_act8_wgrad(int64_t rows, int64_t cols, int64_t out_cols, int dtype, int sm_count)
{
    if (rows == 0 || out_cols == 0) return 0;
    // Which operands are laid out depends on the call's addresses (a launch takes more rows when fewer are): room for every choice.
    Plan p = {};
    int64_t lay = 0;
    for (int k = 0; k < 8; ++k) {
        p = make_plan(rows, cols, out_cols, dtype, (k & 1) != 0, (k & 2) != 0, (k & 4) != 0, sm_count > 0 ? sm_count : 148);
        const int64_t b = p.terms_bytes + p.kept_bytes + p.scales_bytes;
        if (b > lay) lay = b;
    }
    return (size_t)(p.slots_bytes + p.bias_bytes + lay);
}

cudaError_t launch_act8_wgrad(const Wgrad8& p, int sm_count, cudaStream_t stream)
{
    const bool acc = p.accumulate != 0;
    cudaError_t e = cudaSuccess;
    if (p.rows == 0) {
        if (acc) return e;
        const int64_t n = p.cols * p.out_cols, m = p.db ? p.out_cols : 0;
        const int64_t want = (n + m + kThreads - 1) / kThreads, most = (int64_t)sm_count * 8;
        launch_begin("k_wgrad_zero", stream);
        e = launch_pdl(k_wgrad_zero, (int)(want < most ? want : most), kThreads, 0, stream, p.dw, n, p.db, m);
        launch_end(stream);
        return e;
    }
    const bool lay_dy = p.dtype != OGQ_BF16 || ((uintptr_t)p.dy & 15) || p.ld_dy % 8 || p.ld_dy >= (int64_t)1 << 39;  // (a tensor map's limit)
    const bool lay_x = ((uintptr_t)p.codes & 15) || p.cols % 16;
    const bool lay_s = ((uintptr_t)p.scales & 3) != 0;
    if (act8_wgrad_is_small(p, lay_dy || lay_x || lay_s || (p.db && p.rows > kBiasRows))) return launch_act8_wgrad_small(p, stream);
    const Plan plan = make_plan(p.rows, p.cols, p.out_cols, p.dtype, lay_dy, lay_x, lay_s, sm_count);
    char* ws = (char*)p.ws;
    float* slots = (float*)ws;
    float* bias_part = (float*)(ws + plan.slots_bytes);
    uint16_t* terms = (uint16_t*)(ws + plan.slots_bytes + plan.bias_bytes);
    int8_t* kept = (int8_t*)((char*)terms + plan.terms_bytes);
    uint8_t* scales_to = (uint8_t*)kept + plan.kept_bytes;

    // One step of bf16 rows: the product's kernel adds up dy for the bias as well.  More: a kernel before it leaves sums over chunks of
    // rows, which the product's kernel joins.  (All of it there, by the warp that TMA leaves free, took the product alone from 430 to 610 us at
    // 16,384 x 4096 x 4096 in a short run, against 30 us for the other kernel.)
    const bool narrow = p.cols <= 128;
    const bool tma_scales = act8_groups(p.cols) % 16 == 0 && (lay_s || ((uintptr_t)p.scales & 15) == 0);
    const bool beside = p.db && p.cols > 0 && p.rows <= kBiasRows && p.dtype == OGQ_BF16;
    // few parts are joined by the product's kernel; one thread's loop over hundreds would hold it up (100,000 x 8 x 8: 62 us)
    const bool joined_there = p.cols > 0 && plan.bias_chunks > 1 && plan.bias_chunks <= kBiasParts;
    if (p.db && !beside) {
        const int size = p.dtype == OGQ_F32 ? 4 : 2;
        const bool vec = ((uintptr_t)p.dy & 15) == 0 && p.ld_dy * size % 16 == 0 && p.ld_dy % 8 == 0 && p.out_cols % 8 == 0;
        WgBias b = {p.dy, p.ld_dy, p.rows, p.out_cols, plan.bias_chunk, bias_part, p.db, plan.bias_chunks, 0, acc};
        b.ctiles = (int)((p.out_cols + (vec ? 255 : 31)) / (vec ? 256 : 32));
        launch_begin("k_wgrad_bias", stream);
        e = with_dtype(p.dtype, [&](auto elem) {
            using E = decltype(elem);
            return vec ? launch_pdl(k_wgrad_bias<E, 8>, b.ctiles * b.chunks, kThreads, 0, stream, b)
                       : launch_pdl(k_wgrad_bias<E, 1>, b.ctiles * b.chunks, kThreads, 0, stream, b);
        });
        launch_end(stream);
        if (e == cudaSuccess && b.chunks > 1 && !joined_there) {
            launch_begin("k_wgrad_bias_join", stream);
            e = launch_pdl(k_wgrad_bias_join, (int)((p.out_cols + 31) / 32), kThreads, 0, stream, b);
            launch_end(stream);
        }
        if (e != cudaSuccess) return e;
    }
    if (p.cols == 0) return e;

    WgArgs a = {};
    a.dw = p.dw;
    a.slots = slots;
    a.cols = p.cols;
    a.out_cols = p.out_cols;
    a.groups = (int)act8_groups(p.cols);
    a.pairs = plan.pairs;
    a.wide = p.cols % 8 == 0 && ((uintptr_t)p.dw & 31) == 0;
    const size_t size = p.dtype == OGQ_F32 ? 4 : 2;
    for (int64_t t = 0; t < p.rows; t += plan.rows) {
        const int64_t rows = p.rows - t < plan.rows ? p.rows - t : plan.rows;
        const int64_t padded = up_to(rows, kStepRows);
        const char* dy = (const char*)p.dy + t * p.ld_dy * size;
        const int8_t* codes = p.codes + t * p.cols;
        const uint8_t* scales = p.scales + t * a.groups;
        if (lay_dy || lay_x || lay_s) {
            WgLayout l = {dy, p.ld_dy, codes, lay_dy ? terms : nullptr, plan.ld_terms, lay_x ? kept : nullptr, plan.ld_kept,
                          scales, lay_s ? scales_to : nullptr, rows * a.groups, rows, padded, p.cols, p.out_cols};
            const int64_t want = ((lay_dy ? padded * plan.ld_terms / 8 : 0) + (lay_x ? rows * plan.ld_kept / 16 : 0) + (lay_s ? rows * a.groups : 0) + kThreads - 1) / kThreads;
            const int ctas = (int)(want < (int64_t)sm_count * 8 ? want : (int64_t)sm_count * 8);
            launch_begin("k_wgrad_layout", stream);
            e = p.dtype == OGQ_F32 ? launch_pdl(k_wgrad_layout<float, 3>, ctas, kThreads, 0, stream, l)
                : p.dtype == OGQ_F16 ? launch_pdl(k_wgrad_layout<__half, 2>, ctas, kThreads, 0, stream, l)
                                     : launch_pdl(k_wgrad_layout<__nv_bfloat16, 1>, ctas, kThreads, 0, stream, l);
            launch_end(stream);
            if (e != cudaSuccess) return e;
        }
        CUtensorMap map_dy, map_x, map_scales;
        const int terms_here = lay_dy ? plan.terms : 1;
        if (!make_map(&map_dy, lay_dy ? (const void*)terms : dy, true, p.out_cols, lay_dy ? terms_here * padded : rows,
                      (lay_dy ? plan.ld_terms : p.ld_dy) * 2, 64) ||
            !make_map(&map_x, lay_x ? kept : codes, false, p.cols, rows, lay_x ? plan.ld_kept : p.cols, narrow ? 64 : 128))
            return cudaErrorInvalidValue;
        // By TMA where it can: a warp's copies of four bytes each take the shared memory pipe a cycle a lane (16,384 x 4096 x 4096: 504 us,
        // with TMA 496).
        a.scales = lay_s ? scales_to : scales;
        a.tma_scales = tma_scales;
        if (!a.tma_scales) map_scales = map_x;  // not used
        else if (!make_map(&map_scales, a.scales, false, a.groups, rows, a.groups, 16)) return cudaErrorInvalidValue;
        a.rows = rows;
        a.steps_x = (int)(padded / kStepRows);
        a.steps = terms_here * a.steps_x;
        a.last_rows = (int)up_to(rows - (int64_t)(a.steps_x - 1) * kStepRows, 16);
        a.accumulate = acc || t > 0;
        a.db = nullptr;
        if (t == 0 && (beside || (p.db && joined_there))) {
            a.db = p.db;
            a.bias_parts = bias_part;
            a.chunks = beside ? 0 : plan.bias_chunks;
            a.dy = lay_dy ? terms : (const uint16_t*)dy;
            a.ld_dy = lay_dy ? plan.ld_terms : p.ld_dy;
            a.dy_rows = rows;
        }
        e = narrow ? launch_product<128>(map_dy, map_x, map_scales, a, stream) : launch_product<256>(map_dy, map_x, map_scales, a, stream);
        if (e != cudaSuccess) return e;
    }
    return e;
}

}  // namespace ogq

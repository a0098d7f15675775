// AdamW over many tensors at once, with states in 32 or in 8 bits.  Per element, each operation rounded to fp32 once:
//
//   g  = k * grad                                   k = grad_scale * factor
//   m' = b1 * m + w1 * g                            w1 = 1 - b1
//   v' = b2 * v + (w2 * g) * g                      w2 = 1 - b2
//   p' = p - (rate * p + a * (m' / d))              d = sqrt(v') * r2 + eps,  rate = lr * decay,  a = lr / c1,  r2 = 1 / sqrt(c2)
//
// (the root and the quotient within two units in the last place).  m' and v' are sums of products that are rounded one by one, not
// fused, so that states held in 8 bits are the same bits for everybody who follows the formulas.
//
// States in 8 bits, in blocks of 256 elements: m is e4m3 times the block's scale max|m'| / 448, v is e5m2 times max v' / 57344.  A
// step moves v by about (1 - b2) v, far less than half the distance of two neighbours on any grid of 8 bits, so rounding to the
// nearest would leave v where it is for good; both states are rounded at random to one of their two neighbours, without bias,
// which keeps their averages.  v gets the wider range: m of a small element beside a large one lies as far below its block's
// largest as the root of v.  A v' above zero never becomes zero: its element's next step would have nothing but its own square
// under the root.
//
// Bound by memory: 28 bytes an element in fp32, 16 with states in 8 bits.
#include <cmath>

#include "mqg_common.cuh"
#include "mqg_list.cuh"
#include "mqg_tma.cuh"
#include "mqg_training.h"
#include "mqg_vector.cuh"

namespace mqg {
namespace {

constexpr int kBlock = 256;                             // elements of a warp, and of a scale
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPerLane = kBlock / 32;
constexpr float kTopM = 448.0f, kTopV = 57344.0f, kLeast = 0x1p-110f;       // below kLeast a block counts as zero

// Tensors of one launch, passed by value: a kernel's parameters hold 32,764 bytes.
template <int CAP> struct AdamwTable {
    int count;
    uint32_t tile_start[CAP + 1];                       // a tile is kWarps blocks
    uint64_t size[CAP];
    void* p[CAP];
    const void* g[CAP];
    void* m[CAP];
    void* v[CAP];
    float* scales[CAP];
    uint64_t first_block[CAP];                          // blocks before the tensor in the whole list
    float decay[CAP];
    uint8_t kind[CAP];                                  // bit 0: p is bf16, bit 1: g is
};
constexpr int kLargeTable = 448;

struct Scalars {
    float b1, w1, b2, w2, eps, lr, c1, c2, grad_scale;
    const float* factor;
    const float* schedule;
    uint32_t step, seed_lo, seed_hi;
};

// What a step takes from the device's memory, and what follows from it.
struct Step {
    float k, a, r2, lr;
    uint32_t t;
    bool skip;
    __device__ __forceinline__ explicit Step(const Scalars& s)
    {
        const bool from_device = s.schedule != nullptr;
        lr = from_device ? __ldcg(s.schedule) : s.lr;
        const float c1 = from_device ? __ldcg(s.schedule + 1) : s.c1, c2 = from_device ? __ldcg(s.schedule + 2) : s.c2;
        t = from_device ? (uint32_t)__ldcg(s.schedule + 3) : s.step;
        const float f = s.factor != nullptr ? __ldcg(s.factor) : 1.0f;
        k = __fmul_rn(s.grad_scale, f);
        skip = !(fabsf(f) > 0.0f && fabsf(f) < INFINITY);
        a = __fdiv_rn(lr, c1);
        r2 = __fdiv_rn(1.0f, __fsqrt_rn(c2));
    }
};

__device__ __forceinline__ void update(float& p, float g, float& m, float& v, const Scalars& s, const Step& st, float rate)
{
    g = __fmul_rn(st.k, g);
    m = __fadd_rn(__fmul_rn(s.b1, m), __fmul_rn(s.w1, g));
    v = __fadd_rn(__fmul_rn(s.b2, v), __fmul_rn(__fmul_rn(s.w2, g), g));
    const float d = __fadd_rn(__fmul_rn(__fsqrt_rn(v), st.r2), s.eps);
    p = __fsub_rn(p, __fadd_rn(__fmul_rn(rate, p), __fmul_rn(st.a, __fdiv_rn(m, d))));
}

// A float of 8 bits: the bits of an fp32 times 2^EXP2, cut off behind bit SHIFT.  The power of two takes the grid's smallest normal
// number to fp32's, so that both have their subnormal numbers in the same place and a code is a shift of fp32's bits.
template <int SHIFT, int EXP2> struct Format {
    // the value of a code's magnitude
    static __device__ __forceinline__ float value(uint32_t code) { return __uint_as_float(code << SHIFT) * exp2f_const(-EXP2); }
    // x >= 0, at most the grid's largest, rounded up if what is cut off and the draw h in 0 .. 2^16 - 1, (h + 1/2) / 2^16 of a
    // step, make a step.  (The largest element of a block comes within two units in the last place of the grid's largest
    // number, from where no draw carries it further, nor leaves it below.)
    static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x * exp2f_const(EXP2)); }
    static __device__ __forceinline__ uint32_t code(uint32_t bits, uint32_t h)
    {
        return (bits + (h << (SHIFT - 16) | 1u << (SHIFT - 17))) >> SHIFT;
    }
    static __device__ __forceinline__ constexpr float exp2f_const(int e)
    {
        return e == 120 ? 0x1p120f : e == -120 ? 0x1p-120f : e == 112 ? 0x1p112f : 0x1p-112f;
    }
};
using FormatM = Format<20, -120>;
using FormatV = Format<21, -112>;

__device__ __forceinline__ float decode_m(uint32_t code, float scale)
{
    return __fmul_rn(__uint_as_float(__float_as_uint(FormatM::value(code & 0x7F)) | (code & 0x80) << 24), scale);
}
__device__ __forceinline__ float decode_v(uint32_t code, float scale) { return __fmul_rn(FormatV::value(code), scale); }

__device__ __forceinline__ uint32_t encode_m(float m, float inverse, uint32_t h)
{
    return FormatM::code(FormatM::bits(__fmul_rn(fabsf(m), inverse)), h) | (m < 0.0f ? 0x80u : 0u);
}
// (also a v that `inverse` takes below fp32's range stays above zero)
__device__ __forceinline__ uint32_t encode_v(float v, float inverse, uint32_t h)
{
    const uint32_t code = FormatV::code(FormatV::bits(__fmul_rn(v, inverse)), (h & 0xFF) << 8 | h >> 8);
    return max(code, min(__float_as_uint(v), inverse > 0.0f ? 1u : 0u));
}

// A block's scale and what its elements are multiplied with for their codes, from its largest magnitude.
__device__ __forceinline__ void scale_of(float most, float top, float& scale, float& inverse)
{
    const bool held = most >= kLeast;
    scale = held ? __fdiv_rn(most, top) : 0.0f;
    inverse = held ? __fdiv_rn(top, most) : 0.0f;
}

// Largest of a warp's non-negative floats.
__device__ __forceinline__ float warp_max(float x) { return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x))); }

__device__ __forceinline__ float load(const void* p, bool bf16, uint64_t i)
{
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store(void* p, bool bf16, uint64_t i, float x)
{
    if (bf16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
    else static_cast<float*>(p)[i] = x;
}

// A warp to a block, lanes side by side.
template <int CAP, bool EIGHT>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ AdamwTable<CAP> tab, const Scalars s)
{
    __shared__ uint4 draws[EIGHT ? kWarps : 1][32];
    const int j = find_in_list<(CAP > 32)>(tab.tile_start, tab.count, blockIdx.x);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint64_t block = (uint64_t)(blockIdx.x - tab.tile_start[j]) * kWarps + warp, e0 = block * kBlock, size = tab.size[j];
    const bool wide_p = !(tab.kind[j] & 1), wide_g = !(tab.kind[j] & 2);
    const float decay = tab.decay[j];
    grid_dependency_wait();
    const Step st(s);
    if (st.skip || e0 >= size) return;
    const uint32_t held = (uint32_t)min((uint64_t)kBlock, size - e0);
    const float rate = __fmul_rn(st.lr, decay);
    float p[kPerLane], g[kPerLane], m[kPerLane], v[kPerLane];
    float scale_m = 0.0f, scale_v = 0.0f;
    if (EIGHT) {
        scale_m = __ldcg(tab.scales[j] + 2 * block);
        scale_v = __ldcg(tab.scales[j] + 2 * block + 1);
    }
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const uint32_t at = lane + 32 * i;
        const uint64_t e = e0 + at;
        p[i] = g[i] = m[i] = v[i] = 0.0f;
        if (at >= held) continue;
        p[i] = load(tab.p[j], !wide_p, e);
        g[i] = load(tab.g[j], !wide_g, e);
        if (EIGHT) {
            m[i] = decode_m(static_cast<const uint8_t*>(tab.m[j])[e], scale_m);
            v[i] = decode_v(static_cast<const uint8_t*>(tab.v[j])[e], scale_v);
        } else {
            m[i] = static_cast<const float*>(tab.m[j])[e];
            v[i] = static_cast<const float*>(tab.v[j])[e];
        }
    }
    float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        update(p[i], g[i], m[i], v[i], s, st, rate);
        const uint32_t at = lane + 32 * i;
        if (at >= held) continue;
        store(tab.p[j], !wide_p, e0 + at, p[i]);
        if (!EIGHT) {
            static_cast<float*>(tab.m[j])[e0 + at] = m[i];
            static_cast<float*>(tab.v[j])[e0 + at] = v[i];
        }
        most_m = fmaxf(most_m, fabsf(m[i]));
        most_v = fmaxf(most_v, v[i]);
    }
    if (!EIGHT) return;
    float inverse_m, inverse_v;
    scale_of(warp_max(most_m), kTopM, scale_m, inverse_m);
    scale_of(warp_max(most_v), kTopV, scale_v, inverse_v);
    if (lane == 0) {
        tab.scales[j][2 * block] = scale_m;
        tab.scales[j][2 * block + 1] = scale_v;
    }
    // lane l draws for the elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3 of the block
    const uint64_t group = (tab.first_block[j] + block) * 32 + lane;
    const RoundKeys keys = make_round_keys({s.seed_lo, s.seed_hi, 0xFFFFFFFFu, st.t});
    uint32_t y[4];
    philox4x32_10((uint32_t)group, (uint32_t)(group >> 32), 0xFFFFFFFFu, st.t, keys, y);
    draws[warp][lane] = make_uint4(y[0], y[1], y[2], y[3]);
    __syncwarp();
    const uint16_t* half = reinterpret_cast<const uint16_t*>(draws[warp]);
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const uint32_t at = lane + 32 * i;
        if (at >= held) continue;
        const uint32_t h = half[(at % 128 / 4) * 8 + at / 128 * 4 + at % 4];
        static_cast<uint8_t*>(tab.m[j])[e0 + at] = (uint8_t)encode_m(m[i], inverse_m, h);
        static_cast<uint8_t*>(tab.v[j])[e0 + at] = (uint8_t)encode_v(v[i], inverse_v, h);
    }
}

uint64_t blocks_of(uint64_t n) { return (n + kBlock - 1) / kBlock; }

template <int CAP> cudaError_t launch_table(const AdamwList& list, int first, int last, uint64_t& blocks, const Scalars& s, cudaStream_t stream)
{
    AdamwTable<CAP> tab;
    uint64_t tiles = 0;
    int k = 0;
    for (int j = first; j < last; ++j, ++k) {
        tab.tile_start[k] = (uint32_t)tiles;
        tab.size[k] = list.size[j];
        tab.p[k] = list.p[j];
        tab.g[k] = list.g[j];
        tab.m[k] = list.m[j];
        tab.v[k] = list.v[j];
        tab.scales[k] = list.scales ? list.scales[j] : nullptr;
        tab.first_block[k] = blocks;
        tab.decay[k] = list.decay ? list.decay[j] : 0.0f;
        tab.kind[k] = (uint8_t)((list.p_dtype[j] == kBf16 ? 1 : 0) | (list.g_dtype[j] == kBf16 ? 2 : 0));
        blocks += blocks_of(list.size[j]);
        tiles += (blocks_of(list.size[j]) + kWarps - 1) / kWarps;
    }
    tab.tile_start[k] = (uint32_t)tiles;
    tab.count = k;
    if (tiles == 0) return cudaSuccess;
    return list.scales ? launch_pdl(adamw_kernel<CAP, true>, (unsigned)tiles, kThreads, stream, tab, s)
                       : launch_pdl(adamw_kernel<CAP, false>, (unsigned)tiles, kThreads, stream, tab, s);
}

}  // namespace

cudaError_t launch_adamw(const AdamwList& list, const AdamwStep& step, cudaStream_t stream)
{
    Scalars s;
    s.b1 = (float)step.beta1;
    s.w1 = (float)(1.0 - step.beta1);
    s.b2 = (float)step.beta2;
    s.w2 = (float)(1.0 - step.beta2);
    s.eps = (float)step.eps;
    s.lr = (float)step.lr;
    s.c1 = (float)(1.0 - std::pow(step.beta1, (double)step.t));
    s.c2 = (float)(1.0 - std::pow(step.beta2, (double)step.t));
    s.grad_scale = step.grad_scale;
    s.factor = step.factor;
    s.schedule = step.schedule;
    s.step = step.t;
    s.seed_lo = (uint32_t)step.seed;
    s.seed_hi = (uint32_t)(step.seed >> 32);
    uint64_t blocks = 0;
    cudaError_t err = cudaSuccess;
    for (int first = 0; first < list.count && err == cudaSuccess; first += kLargeTable) {
        const int last = list.count - first > kLargeTable ? first + kLargeTable : list.count, n = last - first;
        err = n <= 16   ? launch_table<16>(list, first, last, blocks, s, stream)
              : n <= 96 ? launch_table<96>(list, first, last, blocks, s, stream)
                        : launch_table<kLargeTable>(list, first, last, blocks, s, stream);
    }
    return err;
}

}  // namespace mqg

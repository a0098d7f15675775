// AdamW over many tensors at once, with states in 32 or in 8 bits.  Per element, each operation rounded to fp32 once:
//
//   g  = k * grad                                   k = grad_scale * factor
//   m' = b1 * m + w1 * g                            w1 = 1 - b1
//   v' = b2 * v + (w2 * g) * g                      w2 = 1 - b2
//   p' = p - (rate * p + a * (m' / d))              d = sqrt(v') * r2 + eps,  rate = lr * decay,  a = lr / c1,  r2 = 1 / sqrt(c2)
//
// (the root and the quotient within two units in the last place, for every v' and d).  m' and v' are sums of products that are rounded
// one by one, not fused, so that states held in 8 bits are the same bits for everybody who follows the formulas.
//
// States in 8 bits, in blocks of 256 elements: m is e4m3 times the block's scale max|m'| / 448, v is e5m2 times max v' / 57344.  A
// step moves v by about (1 - b2) v, far less than half the distance of two neighbours on any grid of 8 bits, so rounding to the
// nearest would leave v where it is for good; both states are rounded at random to one of their two neighbours, without bias,
// which keeps their averages.  v gets the wider range: m of a small element beside a large one lies as far below its block's
// largest as the root of v.  A v' above zero never becomes zero: its element's next step would have nothing but its own square
// under the root.
//
// In 32 bits bound by memory, 28 bytes an element in fp32: 25 M elements in 106 us, 1.02 of the copy rate.  In 8 bits, 14 bytes with
// bf16 gradients, by instructions, 60 an element: 100 M in 250 us after an idle moment (0.87 of the copy rate), 264 to 275 at the power
// limit.  A block's inputs come by way of shared memory while the one before is computed, which took 288 us to 267.
#include <cuda_fp16.h>

#include <cmath>

#include "mqg_async.cuh"
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
template <int CAP, bool EIGHT> struct AdamwTable {
    int count;
    uint32_t tile_start[CAP + 1];                       // a tile is the blocks of a CTA
    uint64_t size[CAP];
    void* p[CAP];
    const void* g[CAP];
    void* m[CAP];
    void* v[CAP];
    float* scales[EIGHT ? CAP : 1];
    uint64_t first_block[EIGHT ? CAP : 1];              // blocks before the tensor in the whole list
    float decay[CAP];
    uint8_t kind[CAP];                                  // bit 0: p is bf16, bit 1: g is, bit 2: all on the boundaries of 4 elements
};
template <bool EIGHT> constexpr int kLargeTable = EIGHT ? 448 : 640;

// Turns of a warp, where there are more than 128 blocks to an SM, five to each of the 24 warps that it holds.  (100 M elements with states in
// 8 bits by 2 / 4 / 8 / 16 turns: 263 / 251 / 257 / 267 us.)
constexpr uint32_t kTurns = 4, kManyBlocks = 148 * 128;

struct Scalars {
    float b1, w1, b2, w2, eps, lr, a, r2, grad_scale, minus_zero;
    const float* factor;
    const float* schedule;
    uint32_t step;
    RoundKeys keys;
};

// lr / c1 and 1 / sqrt(c2), each operation rounded; the same on the host and on the device.
__host__ __device__ inline float step_size(float lr, float c1)
{
#ifdef __CUDA_ARCH__
    return __fdiv_rn(lr, c1);
#else
    return lr / c1;
#endif
}
__host__ __device__ inline float reciprocal_root(float c2)
{
#ifdef __CUDA_ARCH__
    return __fdiv_rn(1.0f, __fsqrt_rn(c2));
#else
    return 1.0f / std::sqrt(c2);
#endif
}

// What a step takes from the device's memory.
struct FromDevice {
    float factor, schedule[4];
    __device__ __forceinline__ explicit FromDevice(const Scalars& s) : factor(s.factor != nullptr ? __ldcg(s.factor) : 1.0f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) schedule[i] = s.schedule != nullptr ? __ldcg(s.schedule + i) : 0.0f;
    }
};

// And what follows from it: to be formed behind a block's loads, which then do not wait for these.
struct Step {
    float k, a, r2, lr;
    uint32_t t;
    bool skip, any;          // any: the root or the quotient of any number (see root, reciprocal)
    __device__ __forceinline__ Step(const Scalars& s, const FromDevice& d) : k(s.grad_scale), a(s.a), r2(s.r2), lr(s.lr), t(s.step), skip(false)
    {
        if (s.factor != nullptr) {
            skip = !(fabsf(d.factor) > 0.0f && fabsf(d.factor) < INFINITY);
            k = __fmul_rn(s.grad_scale, d.factor);
        }
        if (s.schedule != nullptr) {
            lr = d.schedule[0];
            a = step_size(lr, d.schedule[1]);
            r2 = reciprocal_root(d.schedule[2]);
            t = (uint32_t)d.schedule[3];
        }
        any = !(s.eps >= 0x1p-38f * r2 && s.eps <= 0x1p60f && r2 <= 0x1p15f);
    }
};

// sqrt(x), x >= 0, within two units in the last place; zero below 2^-126, which takes 2^-63 r2 from d at most: below a quarter of d's last
// place where eps is 2^-38 r2 or more.
__device__ __forceinline__ float root(float x)
{
    float r;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / d within one unit in the last place, d < 2^126 or infinite (d is sqrt(v') * r2 + eps, below 2^80 with eps up to 2^60 and r2 up to 2^15).
__device__ __forceinline__ float reciprocal(float d)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    return r;
}

// The same without those limits, and the quotient (its reciprocal would leave fp32's normal numbers).
__device__ __forceinline__ float root_of_any(float x)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float quotient_of_any(float m, float d)
{
    float r;
    asm("div.full.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(d));
    return r;
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// The product of two pairs, rounded, in a form that no later sum is fused with (a packed multiplication is, whatever the source
// says of its rounding): a sum with -0, which the compiler does not know.
__device__ __forceinline__ float2 times(float2 a, float2 b, float minus_zero) { return __ffma2_rn(a, b, both(minus_zero)); }

// The step of two elements, by packed instructions, which round as the single ones do.
__device__ __forceinline__ void update2(float* p, const float* g_in, float* m, float* v, const Scalars& s, const Step& st, float rate)
{
    const float z = s.minus_zero;
    const float2 g = times(both(st.k), make_float2(g_in[0], g_in[1]), z), old = make_float2(p[0], p[1]);
    const float2 m2 = __fadd2_rn(times(both(s.b1), make_float2(m[0], m[1]), z), times(both(s.w1), g, z));
    const float2 v2 = __fadd2_rn(times(both(s.b2), make_float2(v[0], v[1]), z), times(times(both(s.w2), g, z), g, z));
    const float2 d = __ffma2_rn(make_float2(root(v2.x), root(v2.y)), both(st.r2), both(s.eps));
    const float2 u = __fmul2_rn(m2, make_float2(reciprocal(d.x), reciprocal(d.y)));
    const float2 less = __ffma2_rn(both(st.a), u, __fmul2_rn(both(rate), old));
    p[0] = old.x - less.x, p[1] = old.y - less.y;
    m[0] = m2.x, m[1] = m2.y;
    v[0] = v2.x, v[1] = v2.y;
}

// The new parameters again, of any v' and d, from the old ones and the new averages.  (For steps whose scalars ask for it: by itself and with
// the old parameters read again, since the registers do not hold both forms side by side.)
__device__ __forceinline__ void parameters_of_any(float (&p)[kPerLane], const float (&m)[kPerLane], const float (&v)[kPerLane], const Scalars& s,
                                                  const Step& st, float rate)
{
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const float u = quotient_of_any(m[i], fmaf(root_of_any(v[i]), st.r2, s.eps));
        p[i] -= fmaf(st.a, u, __fmul_rn(rate, p[i]));
    }
}

// A float of 8 bits: the bits of an fp32 times 2^EXP2, cut off behind bit SHIFT.  The power of two takes the grid's smallest normal
// number to fp32's, so that both have their subnormal numbers in the same place and a code is a shift of fp32's bits.
template <int SHIFT, int EXP2> struct Format {
    // x >= 0, at most the grid's largest, rounded up if what is cut off and the draw h in 0 .. 2^16 - 1, (h + 1/2) / 2^16 of a
    // step, make a step.  (The largest element of a block comes within two units in the last place of the grid's largest
    // number, from where no draw carries it further, nor leaves it below.)
    static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x * (EXP2 == -120 ? 0x1p-120f : 0x1p-112f)); }
    static __device__ __forceinline__ uint32_t code(uint32_t bits, uint32_t h)
    {
        return (bits + (h << (SHIFT - 16) | 1u << (SHIFT - 17))) >> SHIFT;
    }
};
using FormatM = Format<20, -120>;
using FormatV = Format<21, -112>;

// (an infinite m times its block's inverse, 0, is a NaN, of which nothing reaches the sign)
__device__ __forceinline__ uint32_t encode_m(float m, float inverse, uint32_t h)
{
    return FormatM::code(FormatM::bits(__fmul_rn(fabsf(m), inverse)), h) & 0x7Fu | (__float_as_uint(m) >> 24 & 0x80u);
}
// (a v of 2^-128 or more never becomes zero, also where `inverse` takes it below fp32's range)
__device__ __forceinline__ uint32_t encode_v(float v, float inverse, uint32_t h)
{
    const uint32_t code = FormatV::code(FormatV::bits(__fmul_rn(v, inverse)), (h & 0xFF) << 8 | h >> 8);
    return max(code, min(__float_as_uint(v), inverse > 0.0f ? 1u << 21 : 0u) >> 21);
}

// Largest magnitude; a NaN among them stays one.
__device__ __forceinline__ float largest(float most, float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(most), "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
// Largest of a warp's non-negative floats (as numbers their bits are in the same order, and a NaN's are above all).
__device__ __forceinline__ float warp_max(float x) { return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x))); }

// A block's two scales, which it stores, and what its elements are multiplied with for their codes.  One division for the warp: lane
// 0 has m's scale, 1 its inverse, 2 and 3 those of v.
__device__ __forceinline__ void new_scales(float most_m, float most_v, float* scales, float& inverse_m, float& inverse_v)
{
    const uint32_t lane = threadIdx.x & 31;
    const float all_m = warp_max(most_m), all_v = warp_max(most_v), most = lane & 2 ? all_v : all_m, top = lane & 2 ? kTopV : kTopM;
    const float q = most < kLeast ? 0.0f : __fdiv_rn(lane & 1 ? top : most, lane & 1 ? most : top);      // (of a NaN: NaN)
    if (lane == 0 || lane == 2) scales[lane >> 1] = q;
    inverse_m = __shfl_sync(0xFFFFFFFFu, q, 1);
    inverse_v = __shfl_sync(0xFFFFFFFFu, q, 3);
}

// The values of two codes of each; all of one block.  fp16 holds the values of both formats, infinities and NaN among them: e5m2 is
// its upper byte.
__device__ __forceinline__ void decode2(uint16_t m, uint32_t half_v, float scale_m, float scale_v, float* to_m, float* to_v)
{
    uint32_t half_m;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(half_m) : "h"(m));
    const float2 x = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2*>(&half_m)), both(scale_m));
    const float2 y = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2*>(&half_v)), both(scale_v));
    to_m[0] = x.x, to_m[1] = x.y;
    to_v[0] = y.x, to_v[1] = y.y;
}

// Four codes in a word, and back.
__device__ __forceinline__ void decode4(uint32_t m, uint32_t v, float scale_m, float scale_v, float* to_m, float* to_v)
{
    decode2((uint16_t)m, __byte_perm(v, 0, 0x1404), scale_m, scale_v, to_m, to_v);
    decode2((uint16_t)(m >> 16), __byte_perm(v, 0, 0x3424), scale_m, scale_v, to_m + 2, to_v + 2);
}

// One half of a word of draws, times 2^p, plus x; `half`: 2^p in the byte that meets that half in a two-way dot product.
__device__ __forceinline__ uint32_t add_draw(uint32_t draws, uint32_t half, uint32_t x) { return __dp2a_lo(draws, half, x); }

// draws: of the four elements, two to a word.
__device__ __forceinline__ void encode4(const float* m, const float* v, float inverse_m, float inverse_v, const uint32_t* draws,
                                        uint32_t& codes_m, uint32_t& codes_v)
{
    uint32_t at_top_m[4], at_top_v[4];
    const uint32_t least = inverse_v > 0.0f ? 1u << 21 : 0u;
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        const float2 x = __fmul2_rn(__fmul2_rn(make_float2(m[j], m[j + 1]), both(inverse_m)), both(0x1p-120f));
        const float2 y = __fmul2_rn(__fmul2_rn(make_float2(v[j], v[j + 1]), both(inverse_v)), both(0x1p-112f));
        const uint32_t h = draws[j / 2], turned = __byte_perm(h, 0, 0x2301);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t bits_m = add_draw(h, i ? 16u << 8 : 16u, __float_as_uint(i ? x.y : x.x));   // (27 bits below the sign)
            const uint32_t bits_v = add_draw(turned, i ? 32u << 8 : 32u, __float_as_uint(i ? y.y : y.x));
            at_top_m[j + i] = __float_as_uint(m[j + i]) & 0x80000000u | bits_m * 16u + 8u * 16u & 0x7FFFFFFFu;
            at_top_v[j + i] = max(bits_v + 16u, min(__float_as_uint(v[j + i]), least)) * 8u;
        }
    }
    codes_m = __byte_perm(__byte_perm(at_top_m[0], at_top_m[1], 0x0073), __byte_perm(at_top_m[2], at_top_m[3], 0x0073), 0x5410);
    codes_v = __byte_perm(__byte_perm(at_top_v[0], at_top_v[1], 0x0073), __byte_perm(at_top_v[2], at_top_v[3], 0x0073), 0x5410);
}

template <bool EIGHT> struct StateType { using type = float; };
template <> struct StateType<true> { using type = uint8_t; };

// One block of one tensor.
struct Block {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* scales;
    uint64_t e0, group0;     // first element; number of the block's first group of draws
    uint32_t held;           // elements of the last block
    float decay;
    uint32_t kind;
    // the warp's block so many turns further on
    __device__ __forceinline__ void advance(uint32_t turns)
    {
        e0 += (uint64_t)turns * (kWarps * kBlock);
        group0 += (uint64_t)turns * (kWarps * 32);
        if (scales != nullptr) scales += (uint64_t)turns * (kWarps * 2);
    }
};

__device__ __forceinline__ void draw(uint64_t group, const Step& st, const RoundKeys& keys, uint32_t (&y)[4])
{
    philox4x32_10((uint32_t)group, (uint32_t)(group >> 32), 0xFFFFFFFFu, st.t, keys, y);   // (no worker's draws of the codec)
}

// Where a lane's elements of a whole block on the boundaries of four elements are: lane l has the elements 4 l .. 4 l + 3 and
// 128 + 4 l .. 128 + 4 l + 3, those it draws for.
template <int P, int G, bool EIGHT> struct Place {
    using Four = typename Word<EIGHT ? 4 : 16>::type;    // of m or v
    typename Element<P>::type* p;
    const typename Element<G>::type* g;
    Four* m;
    Four* v;
    float* scales;
    __device__ __forceinline__ explicit Place(const Block& b)
    {
        const uint64_t e = b.e0 + (threadIdx.x & 31) * 4;
        p = static_cast<typename Element<P>::type*>(b.p) + e;
        g = static_cast<const typename Element<G>::type*>(b.g) + e;
        m = static_cast<Four*>(b.m) + e / 4;
        v = static_cast<Four*>(b.v) + e / 4;
        scales = b.scales;
    }
    __device__ __forceinline__ void advance()
    {
        p += kWarps * kBlock;
        g += kWarps * kBlock;
        m += kWarps * kBlock / 4;
        v += kWarps * kBlock / 4;
        if (EIGHT) scales += kWarps * 2;
    }
};

// What a lane has of it.
template <int P, int G, bool EIGHT> struct Inputs {
    using Four = typename Place<P, G, EIGHT>::Four;
    Packed<P, 4> p[2];
    Packed<G, 4> g[2];
    Four m[2], v[2];
    float scale_m, scale_v;

    __device__ __forceinline__ explicit Inputs(const Place<P, G, EIGHT>& at)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            p[k].load(at.p + 128 * k);
            g[k].load(at.g + 128 * k);
            m[k] = __ldcg(at.m + 32 * k);
            v[k] = __ldcg(at.v + 32 * k);
        }
    }

    // The same by way of shared memory: asynchronous copies, of each lane's own but for the scales.
    struct Stage {
        Packed<P, 4> p[2][32];
        Packed<G, 4> g[2][32];
        Four m[2][32], v[2][32];
        float scales[2];
    };
    // The block `ahead` turns further on.
    static __device__ __forceinline__ void fetch(const Place<P, G, EIGHT>& at, int ahead, Stage& to)
    {
        const uint32_t lane = threadIdx.x & 31;
        const int skip = ahead * kWarps;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            copy_async<4 * kElemBytes<P>>(&to.p[k][lane], at.p + 128 * k + skip * kBlock);
            copy_async<4 * kElemBytes<G>>(&to.g[k][lane], at.g + 128 * k + skip * kBlock);
            copy_async<sizeof(Four)>(&to.m[k][lane], at.m + 32 * k + skip * (kBlock / 4));
            copy_async<sizeof(Four)>(&to.v[k][lane], at.v + 32 * k + skip * (kBlock / 4));
        }
        if (lane < 2) copy_async<4>(&to.scales[lane], at.scales + lane + skip * 2);
    }
    __device__ __forceinline__ explicit Inputs(const Stage& from)
    {
        const uint32_t lane = threadIdx.x & 31;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            p[k] = from.p[k][lane];
            g[k] = from.g[k][lane];
            m[k] = from.m[k][lane];
            v[k] = from.v[k][lane];
        }
        scale_m = from.scales[0];
        scale_v = from.scales[1];
    }
};

template <int P, int G, bool EIGHT>
__device__ __forceinline__ void step_vectors(const Place<P, G, EIGHT>& at, uint64_t group, Inputs<P, G, EIGHT>& in, const Scalars& s,
                                             const Step& st, float rate)
{
    float p[8], g[8], m[8], v[8];
    uint32_t y[4];
    if (EIGHT) draw(group, st, s.keys, y);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        widen_to<P, 4>(in.p[k], p + 4 * k);
        widen_to<G, 4>(in.g[k], g + 4 * k);
        if constexpr (EIGHT) {
            decode4(in.m[k], in.v[k], in.scale_m, in.scale_v, m + 4 * k, v + 4 * k);
        } else {
            *reinterpret_cast<uint4*>(m + 4 * k) = in.m[k];
            *reinterpret_cast<uint4*>(v + 4 * k) = in.v[k];
        }
    }
    float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        update2(p + i, g + i, m + i, v + i, s, st, rate);
        if (EIGHT) {
            most_m = largest(most_m, m[i], m[i + 1]);
            most_v = largest(most_v, v[i], v[i + 1]);
        }
    }
    if (st.any) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            in.p[k].load(at.p + 128 * k);
            widen_to<P, 4>(in.p[k], p + 4 * k);
        }
        parameters_of_any(p, m, v, s, st, rate);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) in.p[k].set(i, p[4 * k + i]);
        in.p[k].store(at.p + 128 * k);
        if constexpr (!EIGHT) {
            at.m[32 * k] = *reinterpret_cast<uint4*>(m + 4 * k);
            at.v[32 * k] = *reinterpret_cast<uint4*>(v + 4 * k);
        }
    }
    if constexpr (EIGHT) {
        float inverse_m, inverse_v;
        new_scales(most_m, most_v, at.scales, inverse_m, inverse_v);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t codes_m, codes_v;
            encode4(m + 4 * k, v + 4 * k, inverse_m, inverse_v, y + 2 * k, codes_m, codes_v);
            at.m[32 * k] = codes_m;
            at.v[32 * k] = codes_v;
        }
    }
}

// Any block, lanes side by side.  WHOLE: it has all of its elements.  draws: 32 words of 16 bytes for this warp.
template <int P, int G, bool EIGHT, bool WHOLE>
__device__ __forceinline__ void step_elements(const Block& b, const Scalars& s, const FromDevice& d, uint4* draws)
{
    using State = typename StateType<EIGHT>::type;
    const uint32_t lane = threadIdx.x & 31;
    const uint64_t first = b.e0 + lane;
    auto* at_p = static_cast<typename Element<P>::type*>(b.p) + first;
    const auto* at_g = static_cast<const typename Element<G>::type*>(b.g) + first;
    auto* at_m = static_cast<State*>(b.m) + first;
    auto* at_v = static_cast<State*>(b.v) + first;
    const auto has = [&](int i) { return WHOLE || lane + 32 * i < b.held; };
    typename Element<P>::type in_p[kPerLane];
    typename Element<G>::type in_g[kPerLane];
    State in_m[kPerLane], in_v[kPerLane];
    float scale_m = 0.0f, scale_v = 0.0f;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        in_p[i] = has(i) ? __ldcg(at_p + 32 * i) : typename Element<P>::type(0.0f);
        in_g[i] = has(i) ? __ldcg(at_g + 32 * i) : typename Element<G>::type(0.0f);
        in_m[i] = has(i) ? __ldcg(at_m + 32 * i) : State(0);
        in_v[i] = has(i) ? __ldcg(at_v + 32 * i) : State(0);
    }
    if (EIGHT) {
        scale_m = __ldcg(b.scales);
        scale_v = __ldcg(b.scales + 1);
    }
    const Step st(s, d);
    if (st.skip) return;
    const float rate = __fmul_rn(st.lr, b.decay);
    float p[kPerLane], g[kPerLane], m[kPerLane], v[kPerLane];
    float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        p[i] = widen(in_p[i]);
        g[i] = widen(in_g[i]);
        if constexpr (!EIGHT) {
            m[i] = in_m[i];
            v[i] = in_v[i];
        } else if (i % 2 == 0) {
            decode2((uint16_t)(in_m[i] | in_m[i + 1] << 8), (uint32_t)in_v[i] << 8 | (uint32_t)in_v[i + 1] << 24, scale_m, scale_v, m + i, v + i);
        }
    }
#pragma unroll
    for (int i = 0; i < kPerLane; i += 2) {
        update2(p + i, g + i, m + i, v + i, s, st, rate);
        if (EIGHT) {
            most_m = largest(most_m, m[i], m[i + 1]);  // (places without elements stay zeros)
            most_v = largest(most_v, v[i], v[i + 1]);
        }
    }
    if (st.any) {
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) p[i] = has(i) ? widen(__ldcg(at_p + 32 * i)) : 0.0f;
        parameters_of_any(p, m, v, s, st, rate);
    }
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        if (!has(i)) continue;
        narrow(p[i], at_p[32 * i]);
        if constexpr (!EIGHT) {
            at_m[32 * i] = m[i];
            at_v[32 * i] = v[i];
        }
    }
    if constexpr (EIGHT) {
        float inverse_m, inverse_v;
        new_scales(most_m, most_v, b.scales, inverse_m, inverse_v);
        uint32_t y[4];
        draw(b.group0 + lane, st, s.keys, y);
        __syncwarp();                                   // the draws of the block before have been read
        draws[lane] = make_uint4(y[0], y[1], y[2], y[3]);
        __syncwarp();
        // element lane + 32 i: group lane / 4 + 8 (i % 4), place 4 (i / 4) + lane % 4
        const uint16_t* half = reinterpret_cast<const uint16_t*>(draws) + (lane / 4) * 8 + lane % 4;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const uint32_t h = half[(i % 4) * 64 + (i / 4) * 4];
            if (!has(i)) continue;
            at_m[32 * i] = (uint8_t)encode_m(m[i], inverse_m, h);
            at_v[32 * i] = (uint8_t)encode_v(v[i], inverse_v, h);
        }
    }
}

// The blocks of a tensor that a warp takes, kWarps apart: `whole` of 256 elements, and perhaps the last one of fewer.
struct Run {
    uint32_t whole, rest;    // rest: elements of the last one; 0: another warp's, or there is none
    __device__ __forceinline__ Run(uint64_t first, uint64_t size, uint32_t turns)
    {
        const uint64_t blocks = size / kBlock, left = blocks > first ? blocks - first : 0;
        whole = (uint32_t)min((left + kWarps - 1) / kWarps, (uint64_t)turns);
        rest = whole < turns && first + (uint64_t)whole * kWarps == blocks ? (uint32_t)(size % kBlock) : 0;
    }
};

constexpr int kStages = 2;
constexpr int kWarpBytes = kStages * sizeof(Inputs<kF32, kF32, true>::Stage);

// States in 8 bits: a block's inputs come by way of shared memory while the one before is computed, since arithmetic and memory
// take about as long; in 32 bits, where memory does, straight to registers.
template <int P, int G, bool EIGHT>
__device__ __forceinline__ void step_run(Block b, const Run& run, const Scalars& s, unsigned char* memory, uint4* draws)
{
    const FromDevice d(s);
    using In = Inputs<P, G, EIGHT>;
    if (!(b.kind & 4)) {
#pragma unroll 1
        for (uint32_t turn = 0; turn < run.whole; ++turn, b.advance(1)) step_elements<P, G, EIGHT, true>(b, s, d, draws);
    } else {
        Place<P, G, EIGHT> at(b);
        uint64_t group = b.group0 + (threadIdx.x & 31);
        if constexpr (EIGHT) {
            auto* stage = reinterpret_cast<typename In::Stage*>(memory);
            if (run.whole > 0) In::fetch(at, 0, stage[0]);
            commit_copies();
            const Step st(s, d);
            const float rate = __fmul_rn(st.lr, b.decay);
            if (!st.skip)
#pragma unroll 1
                for (uint32_t turn = 0; turn < run.whole; ++turn) {
                    __syncwarp();                       // the scales of the stage that is filled now have been read
                    if (turn + 1 < run.whole) In::fetch(at, 1, stage[(turn + 1) & 1]);
                    commit_copies();
                    wait_copies<1>();
                    __syncwarp();
                    In in(stage[turn & 1]);
                    step_vectors<P, G, EIGHT>(at, group, in, s, st, rate);
                    at.advance();
                    group += kWarps * 32;
                }
            wait_copies<0>();
        } else {
#pragma unroll 1
            for (uint32_t turn = 0; turn < run.whole; ++turn) {
                In in(at);
                const Step st(s, d);
                if (st.skip) return;
                step_vectors<P, G, EIGHT>(at, group, in, s, st, __fmul_rn(st.lr, b.decay));
                at.advance();
            }
        }
        b.advance(run.whole);
    }
    if (run.rest != 0) step_elements<P, G, EIGHT, false>(b, s, d, draws);
}

// A warp to a block, `turns` times; a tile is the blocks that a CTA takes.  (Three CTAs to an SM: with four, 64 registers spill, for the
// same time.)
template <int CAP, bool EIGHT>
__global__ void __launch_bounds__(kThreads, 3) adamw_kernel(const __grid_constant__ AdamwTable<CAP, EIGHT> tab, const __grid_constant__ Scalars s, uint32_t turns)
{
    __shared__ __align__(16) unsigned char stages[EIGHT ? kWarps : 1][EIGHT ? kWarpBytes : 16];
    __shared__ uint4 draws[EIGHT ? kWarps : 1][32];
    const int j = find_in_list<(CAP > 32)>(tab.tile_start, tab.count, blockIdx.x);
    const uint32_t warp = threadIdx.x >> 5;
    const uint64_t first = (uint64_t)(blockIdx.x - tab.tile_start[j]) * (kWarps * turns) + warp;
    const Run run(first, tab.size[j], turns);
    Block b;
    b.p = tab.p[j];
    b.g = tab.g[j];
    b.m = tab.m[j];
    b.v = tab.v[j];
    b.scales = EIGHT ? tab.scales[j] + 2 * first : nullptr;
    b.e0 = first * kBlock;
    b.group0 = EIGHT ? (tab.first_block[j] + first) * 32 : 0;
    b.held = run.rest;
    b.decay = tab.decay[j];
    b.kind = tab.kind[j];
    unsigned char* memory = stages[EIGHT ? warp : 0];
    uint4* of_warp = draws[EIGHT ? warp : 0];
    grid_dependency_wait();
    if (b.kind & 1) b.kind & 2 ? step_run<kBf16, kBf16, EIGHT>(b, run, s, memory, of_warp) : step_run<kBf16, kF32, EIGHT>(b, run, s, memory, of_warp);
    else b.kind & 2 ? step_run<kF32, kBf16, EIGHT>(b, run, s, memory, of_warp) : step_run<kF32, kF32, EIGHT>(b, run, s, memory, of_warp);
}

uint64_t blocks_of(uint64_t n) { return (n + kBlock - 1) / kBlock; }

// `blocks`: before tensor `first` in the whole list; moved on.
template <int CAP, bool EIGHT>
cudaError_t launch_table(const AdamwList& list, int first, int last, uint64_t& blocks, const Scalars& s, uint32_t turns, cudaStream_t stream)
{
    AdamwTable<CAP, EIGHT> tab;
    uint64_t tiles = 0;
    int k = 0;
    for (int j = first; j < last; ++j, ++k) {
        const int half_p = list.p_dtype[j] == kBf16, half_g = list.g_dtype[j] == kBf16;
        const auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
        const uintptr_t off = (at(list.p[j]) << half_p | at(list.g[j]) << half_g) & 15;       // of 4 bf16 elements: 8 bytes
        const uintptr_t state_off = (at(list.m[j]) | at(list.v[j])) & (EIGHT ? 3 : 15);
        const uint64_t n_blocks = blocks_of(list.size[j]);
        tab.tile_start[k] = (uint32_t)tiles;
        tab.size[k] = list.size[j];
        tab.p[k] = list.p[j];
        tab.g[k] = list.g[j];
        tab.m[k] = list.m[j];
        tab.v[k] = list.v[j];
        if constexpr (EIGHT) {
            tab.scales[k] = list.scales[j];
            tab.first_block[k] = blocks;
        }
        tab.decay[k] = list.decay ? list.decay[j] : 0.0f;
        tab.kind[k] = (uint8_t)(half_p | half_g << 1 | ((off | state_off) == 0) << 2);
        blocks += n_blocks;
        tiles += turns == 1 ? (n_blocks + kWarps - 1) / kWarps : (n_blocks + kWarps * kTurns - 1) / (kWarps * kTurns);
    }
    tab.tile_start[k] = (uint32_t)tiles;
    tab.count = k;
    if (tiles == 0) return cudaSuccess;
    return launch_pdl(adamw_kernel<CAP, EIGHT>, (unsigned)tiles, kThreads, stream, tab, s, turns);
}

template <bool EIGHT> cudaError_t launch_list(const AdamwList& list, const Scalars& s, cudaStream_t stream)
{
    uint64_t blocks = 0;
    for (int j = 0; j < list.count; ++j) blocks += blocks_of(list.size[j]);
    const uint32_t turns = blocks > (uint64_t)kManyBlocks ? kTurns : 1;
    blocks = 0;
    cudaError_t err = cudaSuccess;
    for (int first = 0; first < list.count && err == cudaSuccess; first += kLargeTable<EIGHT>) {
        const int last = list.count - first > kLargeTable<EIGHT> ? first + kLargeTable<EIGHT> : list.count, n = last - first;
        err = n <= 16    ? launch_table<16, EIGHT>(list, first, last, blocks, s, turns, stream)
              : n <= 96  ? launch_table<96, EIGHT>(list, first, last, blocks, s, turns, stream)
              : n <= 320 ? launch_table<320, EIGHT>(list, first, last, blocks, s, turns, stream)
                         : launch_table<kLargeTable<EIGHT>, EIGHT>(list, first, last, blocks, s, turns, stream);
    }
    return err;
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
    s.a = step_size(s.lr, (float)(1.0 - std::pow(step.beta1, (double)step.t)));
    s.r2 = reciprocal_root((float)(1.0 - std::pow(step.beta2, (double)step.t)));
    s.grad_scale = step.grad_scale;
    s.minus_zero = -0.0f;
    s.factor = step.factor;
    s.schedule = step.schedule;
    s.step = step.t;
    for (uint32_t r = 0; r < 10; ++r) {
        s.keys.k0[r] = (uint32_t)step.seed + r * 0x9E3779B9u;
        s.keys.k1[r] = (uint32_t)(step.seed >> 32) + r * 0xBB67AE85u;
    }
    return list.scales ? launch_list<true>(list, s, stream) : launch_list<false>(list, s, stream);
}

}  // namespace mqg

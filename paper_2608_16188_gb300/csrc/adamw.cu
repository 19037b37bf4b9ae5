// adamw.cu -- one AdamW step (decoupled weight decay) over many tensors at once: the
// update that the gradients of an adaptation step are for (Section 3.1 adapts the
// visual experts and their gating network).
//
//   g' = grad_scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//   p  = p (1 - r wd) - r (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps),  r = lr lr_scale
//
// Moments in fp32, or in 8 bits: m and sqrt(v) as e4m3 values times an fp32 scale for
// each block of 256 elements, the block's largest magnitude / 448.  e4m3 keeps three
// bits of mantissa, while an average moves by 1 - b2 = 0.1% a step: rounded to nearest
// it would stand still, so both are rounded up or down at random with the value as the
// mean.  The random numbers are a hash of (seed, step, tensor, element).  sqrt(v)
// rather than v: e4m3's range, 2^17 from the block's largest value down, then covers
// that range of gradients and not its square root.  Below it the two roundings, each on a
// grid of its own, must not part: m becomes a whole step now and then, and over a sqrt(v)
// of 0 that would be an update of m / eps.  So a positive sqrt(v) is never rounded to 0
// but to a step at least, which bounds |m| / sqrt(v) by the block's own ratio of the two
// scales; such elements take shorter steps than with fp32 moments.
//
// A warp takes two blocks of 256 elements, 8 a lane of each: 16-byte loads of bf16, all
// in flight at once, a block's largest magnitude by one warp reduction, one pass over
// everything.  With 8-bit moments (10 bytes an element) the instructions weigh as much
// as the bytes: 54 an element fill the card's issue slots at the memory's rate.  So the
// arithmetic is packed, and what only rare blocks need is behind a warp-wide branch: the
// rounding below e4m3's normal range, NaN, and square roots of subnormal numbers.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "around.cuh"

namespace vmoe {

namespace {

// Most warps a CTA, and one CTA an SM, 128 registers a thread: 530 us for 302 M bf16
// elements with 8-bit moments (85% of the measured copy rate), 165 us for 38 M with fp32
// moments and a master copy.  Two CTAs of 8 warps: 577 and 166; one of 12 or 18: 581 and
// 696; three of 6: 733.  Fewer pairs than 16 an SM are dealt over all SMs.
constexpr int WARPS = 16;

struct Entry {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    uint32_t whole, rest;  // pairs of whole blocks, and elements behind them
    float lr_scale, decay;
    uint32_t key;  // the tensor's place among the call's, hashed
    int kind;      // bits: fp32 parameters (1), fp32 gradients (2), 8-bit moments (4), master (8)
    __device__ __forceinline__ long long numel() const { return (long long)whole * 512 + rest; }
};
enum { P32 = 1, G32 = 2, S8 = 4, MST = 8 };

// The tensors of a launch, passed by value: `first` is the first pair of blocks of each,
// counted over the launch.
template <int MAX>
struct Table {
    int n;
    bool runs;  // CTAs take runs of pairs
    uint32_t pairs;
    uint32_t first[MAX];
    Entry e[MAX];
};

struct Consts {
    float lr, b1, b2, c1, c2, eps, log_b1, log_b2, zero;  // c1 = 1 - b1, c2 = 1 - b2
    int step;
    uint32_t seed_key;
    const int32_t *step_dev;
    const float *lr_dev, *grad_scale;
};

// What all elements of a tensor share.
struct Rates {
    float keep, rate, root_scale, gs;  // 1 - r wd, r / (1 - b1^t), 1 / sqrt(1 - b2^t), grad_scale
    uint32_t key;
};

// Eight elements as they lie in memory.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(f32x2 (&o)[4]) const {
        o[0] = bf16x2_to_f32x2(v.x);
        o[1] = bf16x2_to_f32x2(v.y);
        o[2] = bf16x2_to_f32x2(v.z);
        o[3] = bf16x2_to_f32x2(v.w);
    }
};
template <>
struct Raw8<float> {
    ulonglong2 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const ulonglong2 *>(p)[0];
        b = reinterpret_cast<const ulonglong2 *>(p)[1];
    }
    __device__ __forceinline__ void get(f32x2 (&o)[4]) const {
        o[0] = a.x;
        o[1] = a.y;
        o[2] = b.x;
        o[3] = b.y;
    }
};

// Eight elements of an array as four pairs of floats; `have` of them where !FULL.
template <bool FULL>
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, int have, f32x2 (&o)[4]) {
    if (FULL) {
        Raw8<__nv_bfloat16> r;
        r.load(p);
        r.get(o);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = pk2(2 * i < have ? __bfloat162float(p[2 * i]) : 0.0f, 2 * i + 1 < have ? __bfloat162float(p[2 * i + 1]) : 0.0f);
    }
}
template <bool FULL>
__device__ __forceinline__ void load8(const float *p, int have, f32x2 (&o)[4]) {
    if (FULL) {
        Raw8<float> r;
        r.load(p);
        r.get(o);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pk2(2 * i < have ? p[2 * i] : 0.0f, 2 * i + 1 < have ? p[2 * i + 1] : 0.0f);
    }
}
template <bool FULL>
__device__ __forceinline__ void store8(__nv_bfloat16 *p, int have, const f32x2 (&v)[4]) {
    if (FULL) {
        *reinterpret_cast<uint4 *>(p) =
            make_uint4(f32x2_to_bf16x2(v[0]), f32x2_to_bf16x2(v[1]), f32x2_to_bf16x2(v[2]), f32x2_to_bf16x2(v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 two = unpk2(v[i >> 1]);
            if (i < have) p[i] = __float2bfloat16_rn(i & 1 ? two.y : two.x);
        }
    }
}
template <bool FULL>
__device__ __forceinline__ void store8(float *p, int have, const f32x2 (&v)[4]) {
    if (FULL) {
        reinterpret_cast<ulonglong2 *>(p)[0] = make_ulonglong2(v[0], v[1]);
        reinterpret_cast<ulonglong2 *>(p)[1] = make_ulonglong2(v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 two = unpk2(v[i >> 1]);
            if (i < have) p[i] = i & 1 ? two.y : two.x;
        }
    }
}
template <bool FULL>
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int have) {
    if (FULL) return *reinterpret_cast<const uint2 *>(p);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < have) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
template <bool FULL>
__device__ __forceinline__ void store_codes(uint8_t *p, int have, uint2 v) {
    if (FULL) {
        *reinterpret_cast<uint2 *>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
    }
}

// Eight e4m3 values times `scale`.
__device__ __forceinline__ void decode(uint2 c, float scale, f32x2 (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t two = (uint16_t)((i < 2 ? c.x : c.y) >> (16 * (i & 1)));
        float lo, hi;
        asm("{\n .reg .b32 t;\n .reg .b16 l, h;\n cvt.rn.f16x2.e4m3x2 t, %2;\n mov.b32 {l, h}, t;\n"
            " cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}"
            : "=f"(lo), "=f"(hi)
            : "h"(two));
        o[i] = mul2(pk2(lo, hi), pk2(scale));
    }
}

__device__ __forceinline__ void square(f32x2 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], v[i]);
}

__device__ __forceinline__ uint32_t e4m3x4(f32x2 lo, f32x2 hi) {
    const float2 a = unpk2(lo), b = unpk2(hi);
    uint32_t r;
    asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n"
        " mov.b32 %0, {l, h};\n}"
        : "=r"(r)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// a rounded to one of the two e4m3 neighbours, `bits` + 8 of 2^20 against the distance to
// the lower one: the bits of the mantissa that e4m3 does not have, 20, are cut off after
// the random number is added (to the magnitude: the sign is the top bit).
__device__ __forceinline__ float dither(float a, uint32_t bits) {
    return __uint_as_float((__float_as_uint(a) + bits + 8u) & 0xfff00000u);
}
// The same for any a.  Below 2^-6, where e4m3's steps stay 2^-9, it is done at 2^-6
// higher, where fp32's first three bits have the same steps.  NaN stays NaN.
__device__ __forceinline__ float dither_any(float a, uint32_t bits) {
    const float low = fabsf(a) < 0.015625f ? 0.015625f : 0.0f * a;  // NaN for NaN
    return copysignf(dither(fabsf(a) + low, bits) - low, a);
}
// sqrt(v): a positive a is one step of e4m3 at least.
__device__ __forceinline__ float dither_root(float a, uint32_t bits) {
    const float q = dither_any(a, bits);
    return a > 0.0f ? fmaxf(q, 0.001953125f) : q;
}
// dither of a positive a from 2^-6 on, with the high half of a hash and as a code: the
// exponent and the first three bits of the mantissa, less the difference of the biases,
// (127 - 7) << 3.  Shifted by 4 they are the top byte, modulo 256, and the random number's
// half is the two bytes in the middle.
__device__ __forceinline__ uint32_t dither_code(float a, uint32_t h) {
    return (__float_as_uint(a) << 4) + __byte_perm(h, 0x40000080u, 0x7324);
}
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// The hash but for its last step, h ^ h >> 16, which is taken with the half it is for:
// 16 times the low or the high half of the result, a multiple of 16 below 2^20.
__device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x9e4a8af7u;
    return (h ^ (h >> 15)) * 0xa6bd2c99u;
}
template <bool HIGH>
__device__ __forceinline__ uint32_t random20(uint32_t h) {
    return (HIGH ? h >> 12 : (h << 4) ^ (h >> 12)) & 0xffff0u;
}

// Three-operand minimum and maximum of magnitudes; a NaN makes the result NaN.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float r;
    asm("min.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The largest magnitude of a block of which this lane holds v, the numbers among it;
// `low` is the least one here (NaN where there is one).
__device__ __forceinline__ uint32_t block_max(const f32x2 (&v)[4], float &low) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 two = unpk2(v[i]);
        f[2 * i] = two.x;
        f[2 * i + 1] = two.y;
    }
    const float top = max3(max3(f[0], f[1], f[2]), max3(f[3], f[4], f[5]), max3(f[6], f[7], f[7]));
    low = min3(min3(f[0], f[1], f[2]), min3(f[3], f[4], f[5]), min3(f[6], f[7], f[7]));
    uint32_t t = __reduce_max_sync(0xffffffffu, __float_as_uint(top));  // NaN above infinity above the rest
    if (t > 0x7f800000u) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[i]));
        t = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
    }
    return t;
}

// The scale of a block with this largest magnitude, and 1 / scale.
__device__ __forceinline__ float2 scale_of(uint32_t t) {
    const float big = __uint_as_float(t);
    if (big < 7.888609052210118e-31f) return make_float2(0.0f, 0.0f);  // 2^-100: 448 / big would overflow
    // 1 / big to nearest: the approximation and one Newton step, where that neither
    // underflows (above 2^125) nor meets an infinity
    float rcp;
    asm("rcp.approx.f32 %0, %1;" : "=f"(rcp) : "f"(big));
    if (t < 0x7e000000u) rcp = fmaf(fmaf(-big, rcp, 1.0f), rcp, rcp);
    return make_float2(big * (1.0f / 448.0f), 448.0f * rcp);
}

// The negative square roots of -v, rounded to nearest: the approximate 1 / sqrt(v) and one
// Newton step on v / sqrt(v).  Where that is no number (0, infinity) or the step
// underflows, sqrtf.  `nv` is -v: with the signs turned the step needs no negation.
template <int NB>
__device__ __forceinline__ void roots(const f32x2 (&nv)[NB][4], f32x2 (&o)[NB][4]) {
    float low = 1.0f;
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) {
        const f32x2 x = nv[i >> 2][i & 3];
        float2 y = unpk2(x);
        asm("{\n .reg .f32 t;\n neg.f32 t, %0;\n rsqrt.approx.ftz.f32 %0, t;\n}" : "+f"(y.x));
        asm("{\n .reg .f32 t;\n neg.f32 t, %0;\n rsqrt.approx.ftz.f32 %0, t;\n}" : "+f"(y.y));
        const f32x2 r = pk2(y.x, y.y), ns = mul2(x, r);
        o[i >> 2][i & 3] = fma2(fma2(ns, ns, x), mul2(r, pk2(0.5f)), ns);
        const float2 two = unpk2(o[i >> 2][i & 3]);
        low = min3(low, two.x, two.y);
    }
    if (__any_sync(0xffffffffu, !(low >= 8.8817841970012523e-16f))) {  // 2^-50
#pragma unroll
        for (int i = 0; i < 4 * NB; ++i) {
            const float2 x = unpk2(nv[i >> 2][i & 3]);
            o[i >> 2][i & 3] = pk2(-sqrtf(-x.x), -sqrtf(-x.y));
        }
    }
}

// a b, which the compiler cannot make one instruction with a sum that follows: it adds a
// zero that it does not know (a product and a sum of packed instructions it does join,
// although both say how they round).
__device__ __forceinline__ f32x2 product(f32x2 a, f32x2 b, const Consts &k) { return fma2(a, b, pk2(k.zero)); }

// The update of NB blocks: p, g, and the moments as values; p and m become the new ones,
// v becomes -v and `root` -sqrt(v).  Every product and sum of the moments is rounded by itself, as a
// sequence of elementary operations would: what an 8-bit moment is rounded to hangs on
// the last bit now and then, and a reference for it is then easily written.
template <int NB>
__device__ __forceinline__ void adam(f32x2 (&p)[NB][4], const f32x2 (&g)[NB][4], f32x2 (&m)[NB][4], f32x2 (&v)[NB][4],
                                     f32x2 (&root)[NB][4], const Rates &r, const Consts &k) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 gi = mul2(g[b][i], pk2(r.gs));
            m[b][i] = add2(product(pk2(k.b1), m[b][i], k), product(pk2(k.c1), gi, k));
            v[b][i] = add2(product(pk2(-k.b2), v[b][i], k), product(pk2(-k.c2), mul2(gi, gi), k));
        }
    roots<NB>(v, root);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 den = fma2(root[b][i], pk2(-r.root_scale), pk2(k.eps));
            p[b][i] = fma2(p[b][i], pk2(r.keep), mul2(mul2(m[b][i], pk2(-r.rate)), rcp2(den)));
        }
}

// m and sqrt(v), given as its negative, of NB blocks to memory in 8 bits.
template <bool FULL, int NB>
__device__ __forceinline__ void store_moments(const Entry &e, const Rates &r, uint32_t block, int have, f32x2 (&m)[NB][4],
                                              f32x2 (&root)[NB][4]) {
    const int lane = threadIdx.x & 31;
    const long long at = (long long)block * 256 + lane * 8;
    bool rare[2 * NB], any = false;
    {
        // lane i computes scale i of the blocks' 2 NB, m's and v's in turn, and stores it
        float low[2 * NB];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
            const uint32_t t = i & 1 ? block_max(root[i >> 1], low[i]) : block_max(m[i >> 1], low[i]);
            if (lane == i) top = t;
        }
        const float2 mine = scale_of(top);
        if (lane < 2 * NB) (lane & 1 ? e.v_scale : e.m_scale)[block + (lane >> 1)] = mine.x;
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
            const float inv = __shfl_sync(0xffffffffu, mine.y, i);
            rare[i] = !(low[i] * inv >= 0.015625f);
            any |= rare[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i & 1)
                    root[i >> 1][j] = mul2(root[i >> 1][j], pk2(-inv));
                else
                    m[i >> 1][j] = mul2(m[i >> 1][j], pk2(inv));
            }
        }
    }
    uint32_t h[NB][8];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) h[b][i] = mix(((uint32_t)at + 256 * b + i) * 0x51f6db5bu + r.key);
    uint2 cm[NB], cv[NB];
    auto codes_m = [&](int b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = unpk2(m[b][i]);
            m[b][i] = pk2(dither(x.x, random20<false>(h[b][2 * i])), dither(x.y, random20<false>(h[b][2 * i + 1])));
        }
        return make_uint2(e4m3x4(m[b][0], m[b][1]), e4m3x4(m[b][2], m[b][3]));
    };
    auto codes_v = [&](int b) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 y = unpk2(root[b][i]);
            w[2 * i] = dither_code(y.x, h[b][2 * i]);
            w[2 * i + 1] = dither_code(y.y, h[b][2 * i + 1]);
        }
        return make_uint2(top_bytes(w[0], w[1], w[2], w[3]), top_bytes(w[4], w[5], w[6], w[7]));
    };
    if (__any_sync(0xffffffffu, any)) {
        // a value in some block lies below 2^-6; only the codes of that block's m or v take the
        // longer way (all four: 541 against 530 us for 302 M elements)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (__any_sync(0xffffffffu, rare[2 * b])) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 x = unpk2(m[b][i]);
                    m[b][i] = pk2(dither_any(x.x, random20<false>(h[b][2 * i])), dither_any(x.y, random20<false>(h[b][2 * i + 1])));
                }
                cm[b] = make_uint2(e4m3x4(m[b][0], m[b][1]), e4m3x4(m[b][2], m[b][3]));
            } else {
                cm[b] = codes_m(b);
            }
            if (__any_sync(0xffffffffu, rare[2 * b + 1])) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 y = unpk2(root[b][i]);
                    root[b][i] = pk2(dither_root(y.x, random20<true>(h[b][2 * i])), dither_root(y.y, random20<true>(h[b][2 * i + 1])));
                }
                cv[b] = make_uint2(e4m3x4(root[b][0], root[b][1]), e4m3x4(root[b][2], root[b][3]));
            } else {
                cv[b] = codes_v(b);
            }
        }
    } else {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            cm[b] = codes_m(b);
            cv[b] = codes_v(b);
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        store_codes<FULL>((uint8_t *)e.m + at + 256 * b, have, cm[b]);
        store_codes<FULL>((uint8_t *)e.v + at + 256 * b, have, cv[b]);
    }
}

// One block of a tensor, the last and ragged one too.
template <typename P, typename G, bool EIGHT, bool MASTER, bool FULL>
__device__ __forceinline__ void update(const Entry &e, const Rates &r, const Consts &k, uint32_t block) {
    const long long at = (long long)block * 256 + (threadIdx.x & 31) * 8;
    const int have = FULL ? 8 : (int)max(0LL, min(8LL, e.numel() - at));
    f32x2 p[1][4], g[1][4], m[1][4], v[1][4], root[1][4];
    load8<FULL>((const G *)e.grad + at, have, g[0]);
    if (EIGHT) {
        decode(load_codes<FULL>((const uint8_t *)e.m + at, have), e.m_scale[block], m[0]);
        decode(load_codes<FULL>((const uint8_t *)e.v + at, have), e.v_scale[block], v[0]);
        square(v[0]);
    } else {
        load8<FULL>((const float *)e.m + at, have, m[0]);
        load8<FULL>((const float *)e.v + at, have, v[0]);
    }
    if (MASTER)
        load8<FULL>(e.master + at, have, p[0]);
    else
        load8<FULL>((const P *)e.param + at, have, p[0]);
    adam<1>(p, g, m, v, root, r, k);
    if (MASTER) store8<FULL>(e.master + at, have, p[0]);
    store8<FULL>((P *)e.param + at, have, p[0]);
    if (EIGHT) {
        store_moments<FULL, 1>(e, r, block, have, m, root);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[0][i] = mul2(v[0][i], pk2(-1.0f));
        store8<FULL>((float *)e.m + at, have, m[0]);
        store8<FULL>((float *)e.v + at, have, v[0]);
    }
}

// A pair of blocks that the tensor ends within.
template <typename P, typename G, bool EIGHT, bool MASTER>
__device__ __forceinline__ void update_last(const Entry &e, const Rates &r, const Consts &k, uint32_t pair) {
#pragma unroll 1
    for (uint32_t b = 2 * pair; b < 2 * pair + 2 && (long long)b * 256 < e.numel(); ++b)
        update<P, G, EIGHT, MASTER, false>(e, r, k, b);
}

// A warp's way through the launch: every step-th pair up to an end.  The tensor is found
// by bisection once and followed from there.
template <int MAX>
struct Walk {
    const Table<MAX> &tab;
    uint32_t b, step, end;
    int at;
    __device__ __forceinline__ Walk(const Table<MAX> &t, uint32_t first, uint32_t by, uint32_t stop)
        : tab(t), b(first), step(by), end(stop), at(0) {
        int hi = t.n;
        while (hi - at > 1) {
            const int mid = (at + hi) >> 1;
            if (t.first[mid] <= b)
                at = mid;
            else
                hi = mid;
        }
    }
    __device__ __forceinline__ bool more() const { return b < end; }
    __device__ __forceinline__ void next() {
        b += step;
        while (at + 1 < tab.n && tab.first[at + 1] <= b) ++at;
    }
    __device__ __forceinline__ const Entry &entry() const { return tab.e[at]; }
    __device__ __forceinline__ uint32_t pair() const { return b - tab.first[at]; }
    __device__ __forceinline__ bool whole() const { return pair() < entry().whole; }
};

struct Common {
    float lr, inv_c1, root_scale, gs;
    uint32_t key;
    __device__ __forceinline__ Rates of(const Entry &e) const {
        const float rate = lr * e.lr_scale;
        return {1.0f - rate * e.decay, rate * inv_c1, root_scale, gs, key + e.key};
    }
};

// What a pair of blocks with 8-bit moments is read as.
template <typename P, typename G>
struct Raw {
    Raw8<P> p[2];
    Raw8<G> g[2];
    uint2 m[2], v[2];
    float m_scale[2], v_scale[2];
    __device__ __forceinline__ void load(const P *param, const Entry &e, uint32_t pair) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const long long at = (long long)pair * 512 + b * 256 + (threadIdx.x & 31) * 8;
            p[b].load(param + at);
            g[b].load((const G *)e.grad + at);
            m[b] = *reinterpret_cast<const uint2 *>((const uint8_t *)e.m + at);
            v[b] = *reinterpret_cast<const uint2 *>((const uint8_t *)e.v + at);
            m_scale[b] = e.m_scale[2 * pair + b];
            v_scale[b] = e.v_scale[2 * pair + b];
        }
    }
};

// 8-bit moments: whole pairs of one kind of tensors, the next one's loads in flight
// while one is computed; leaves `w` at the first pair that is something else.
template <typename P, typename G, bool MASTER, int MAX>
__device__ __forceinline__ void run_eight(Walk<MAX> &w, const Common &c, const Consts &k, int kind) {
    typedef std::conditional_t<MASTER, float, P> S;  // what the update works on
    auto source = [](const Entry &e) { return (const S *)(MASTER ? (void *)e.master : e.param); };
    if (!w.whole()) {
        update_last<P, G, true, MASTER>(w.entry(), c.of(w.entry()), k, w.pair());
        w.next();
        return;
    }
    Raw<S, G> raw;
    raw.load(source(w.entry()), w.entry(), w.pair());
    for (bool go = true; go;) {
        const Entry &e = w.entry();
        const uint32_t pair = w.pair();
        const Rates r = c.of(e);
        const Raw<S, G> now = raw;
        w.next();
        go = w.more() && w.entry().kind == kind && w.whole();
        if (go) raw.load(source(w.entry()), w.entry(), w.pair());
        f32x2 p[2][4], g[2][4], m[2][4], v[2][4], root[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            now.p[b].get(p[b]);
            now.g[b].get(g[b]);
            decode(now.m[b], now.m_scale[b], m[b]);
            decode(now.v[b], now.v_scale[b], v[b]);
            square(v[b]);
        }
        adam<2>(p, g, m, v, root, r, k);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const long long at = (long long)pair * 512 + b * 256 + (threadIdx.x & 31) * 8;
            if (MASTER) store8<true>(e.master + at, 8, p[b]);
            store8<true>((P *)e.param + at, 8, p[b]);
        }
        store_moments<true, 2>(e, r, 2 * pair, 8, m, root);
    }
}

template <typename P, typename G, bool MASTER, int MAX>
__device__ __forceinline__ void run_f32(Walk<MAX> &w, const Common &c, const Consts &k) {
    const Entry &e = w.entry();
    const Rates r = c.of(e);
    if (w.whole()) {
        update<P, G, false, MASTER, true>(e, r, k, 2 * w.pair());
        update<P, G, false, MASTER, true>(e, r, k, 2 * w.pair() + 1);
    } else {
        update_last<P, G, false, MASTER>(e, r, k, w.pair());
    }
    w.next();
}

template <int MAX>
__global__ void __launch_bounds__(32 * WARPS, 1)
adamw_kernel(const __grid_constant__ Table<MAX> tab, const Consts k) {
    pdl_wait();
    Common c;
    c.gs = k.grad_scale ? *k.grad_scale : 1.0f;
    if (!isfinite(c.gs)) return;  // an overflowed gradient: the step is left out
    const int t = max(1, k.step + (k.step_dev ? *k.step_dev : 0));
    c.lr = k.lr * (k.lr_dev ? *k.lr_dev : 1.0f);
    c.inv_c1 = -1.0f / expm1f((float)t * k.log_b1);
    c.root_scale = 1.0f / sqrtf(-expm1f((float)t * k.log_b2));
    c.key = k.seed_key + (uint32_t)t * 0x339cd49bu;
    typedef __nv_bfloat16 H;
    const uint32_t warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    uint32_t first = blockIdx.x * warps + warp, step = gridDim.x * warps, end = tab.pairs;
    if (tab.runs) {
        first = (uint32_t)((uint64_t)tab.pairs * blockIdx.x / gridDim.x) + warp;
        end = (uint32_t)((uint64_t)tab.pairs * (blockIdx.x + 1) / gridDim.x);
        step = warps;
    }
    for (Walk<MAX> w(tab, first, step, end); w.more();) {
        const int kind = w.entry().kind;
        switch (kind) {
            case P32 | G32: run_f32<float, float, false>(w, c, k); break;
            case 0: run_f32<H, H, false>(w, c, k); break;
            case MST: run_f32<H, H, true>(w, c, k); break;
            case G32: run_f32<H, float, false>(w, c, k); break;
            case G32 | MST: run_f32<H, float, true>(w, c, k); break;
            case P32 | G32 | S8: run_eight<float, float, false>(w, c, k, kind); break;
            case S8: run_eight<H, H, false>(w, c, k, kind); break;
            case MST | S8: run_eight<H, H, true>(w, c, k, kind); break;
            case G32 | S8: run_eight<H, float, false>(w, c, k, kind); break;
            default: run_eight<H, float, true>(w, c, k, kind); break;  // G32 | S8 | MST
        }
    }
}

constexpr int SMALL = 40, LARGE = 380;  // tables of 3.4 and 32 KB; a launch takes at most 32764 B
static_assert(sizeof(Table<LARGE>) + sizeof(Consts) <= 32764, "a launch's arguments");

template <int MAX>
int launch_table(const vmoe_adamw_tensor *tensors, int n, int base, uint32_t pairs, const Consts &k, cudaStream_t s) {
    Table<MAX> tab;
    tab.n = 0;
    tab.pairs = pairs;
    uint32_t at = 0;
    bool eight = false;
    for (int i = 0; i < n; ++i) {
        const vmoe_adamw_tensor &x = tensors[i];
        if (x.numel == 0) continue;
        eight |= x.state == VMOE_STATE_E4M3;
        Entry &e = tab.e[tab.n];
        tab.first[tab.n++] = at;
        at += (uint32_t)((x.numel + 511) / 512);
        e.param = x.param;
        e.grad = x.grad;
        e.m = x.m;
        e.v = x.v;
        e.m_scale = x.m_scale;
        e.v_scale = x.v_scale;
        e.master = x.master;
        e.whole = (uint32_t)(x.numel / 512);
        e.rest = (uint32_t)(x.numel % 512);
        e.lr_scale = x.lr_scale;
        e.decay = x.weight_decay;
        e.key = (uint32_t)(base + i) * 0x5e4087b3u;
        e.kind = (x.param_dtype == VMOE_F32 ? P32 : 0) | (x.grad_dtype == VMOE_F32 ? G32 : 0) |
                 (x.state == VMOE_STATE_E4M3 ? S8 : 0) | (x.master ? MST : 0);
    }
    const uint32_t sms = (uint32_t)num_sms(), warps = std::min<uint32_t>(WARPS, (pairs + sms - 1) / sms);
    const uint32_t ctas = std::min((pairs + warps - 1) / warps, sms);
    // Warps dealt over all pairs in turn stay in one part of every array; of short tensors
    // each pair is another one's, and a CTA takes a run of pairs instead.  Tensors of 20000
    // elements, fp32 moments: 30 us in runs, 36 dealt (300 of them); of 147000, with a
    // master copy: 127 and 123 (192); 8-bit moments: 60 and 66; of 885000: 59 both.
    tab.runs = pairs < (uint64_t)tab.n * (eight ? 1024 : 128);
    return launch_kernel(adamw_kernel<MAX>, dim3(ctas), dim3(32 * warps), 0, s, tab, k);
}

}  // namespace

int launch_adamw(int n, const vmoe_adamw_tensor *tensors, const vmoe_adamw_config *c, cudaStream_t s) {
    Consts k;
    k.lr = (float)c->lr;
    k.b1 = (float)c->beta1;
    k.b2 = (float)c->beta2;
    k.c1 = (float)(1.0 - c->beta1);
    k.c2 = (float)(1.0 - c->beta2);
    k.eps = (float)c->eps;
    k.log_b1 = (float)log(c->beta1);
    k.log_b2 = (float)log(c->beta2);
    k.zero = 0.0f;
    k.step = c->step;
    k.seed_key = c->seed * 0xe32a5e87u;
    k.step_dev = c->step_dev;
    k.lr_dev = c->lr_dev;
    k.grad_scale = c->grad_scale;
    for (int base = 0; base < n;) {
        int m = 0;
        uint64_t pairs = 0;
        while (base + m < n && m < LARGE) {
            const uint64_t more = ((uint64_t)tensors[base + m].numel + 511) / 512;
            if (pairs + more > 0x7fffffffu) break;
            pairs += more;
            ++m;
        }
        if (pairs) {
            trace_before(s, "adamw");
            const int st = m <= SMALL ? launch_table<SMALL>(tensors + base, m, base, (uint32_t)pairs, k, s)
                                      : launch_table<LARGE>(tensors + base, m, base, (uint32_t)pairs, k, s);
            trace_after(s);
            if (st != VMOE_OK) return st;
        }
        base += m;
    }
    return VMOE_OK;
}

}  // namespace vmoe

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
// the gradients' range and not its square root.
//
// A warp takes a block of 256 elements, 8 a lane: 16-byte loads of bf16, the block's
// largest magnitude by one warp reduction, one pass over everything.
#include <math.h>

#include <algorithm>

#include "common.cuh"

namespace vmoe {

namespace {

constexpr int AT = 256;  // threads a CTA

struct Entry {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    long long numel;
    float lr_scale, decay;
    uint32_t key;  // the tensor's place among the call's, hashed
    int kind;      // bits: fp32 parameters (1), fp32 gradients (2), 8-bit moments (4), master (8)
};
enum { P32 = 1, G32 = 2, S8 = 4, MST = 8 };

// The tensors of a launch, passed by value: `first` is the first block of 256 of each,
// counted over the launch.
template <int MAX>
struct Table {
    int n;
    uint32_t blocks;
    uint32_t first[MAX];
    Entry e[MAX];
};

struct Consts {
    float lr, b1, b2, c1, c2, eps, log_b1, log_b2;  // c1 = 1 - b1, c2 = 1 - b2
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

template <typename T>
__device__ __forceinline__ void load8(const T *p, bool full, int have, float (&o)[8]);
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16 *p, bool full, int have, float (&o)[8]) {
    if (full) {
        bf16x8_to_f32(*reinterpret_cast<const uint4 *>(p), o);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = i < have ? __bfloat162float(p[i]) : 0.0f;
    }
}
template <>
__device__ __forceinline__ void load8<float>(const float *p, bool full, int have, float (&o)[8]) {
    if (full) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
        o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = i < have ? p[i] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, bool full, int have, const float (&v)[8]);
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16 *p, bool full, int have, const float (&v)[8]) {
    if (full) {
        *reinterpret_cast<uint4 *>(p) = f32_to_bf16x8(v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = __float2bfloat16_rn(v[i]);
    }
}
template <>
__device__ __forceinline__ void store8<float>(float *p, bool full, int have, const float (&v)[8]) {
    if (full) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = v[i];
    }
}

// Eight e4m3 values times `scale`.
__device__ __forceinline__ void load_e4m3(const uint8_t *p, bool full, int have, float scale, float (&o)[8]) {
    uint32_t w[2] = {0, 0};
    if (full) {
        const uint2 r = *reinterpret_cast<const uint2 *>(p);
        w[0] = r.x;
        w[1] = r.y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t two = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
        float lo, hi;
        asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}" : "=f"(lo), "=f"(hi) : "r"(h));
        o[2 * i] = lo * scale;
        o[2 * i + 1] = hi * scale;
    }
}

__device__ __forceinline__ uint16_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// |v| inv rounded to one of the two e4m3 neighbours, 20 bits of `bits` against the
// distance to the lower one.  The bits of the mantissa that e4m3 does not have are cut
// off after the random number is added; below 2^-6, where e4m3's steps stay 2^-9, that is
// done at 2^-6 higher, where fp32's first three bits have the same steps.  NaN stays NaN.
__device__ __forceinline__ float dither(float v, float inv, uint32_t bits) {
    const float a = fabsf(v) * inv;
    const float low = a < 0.015625f ? 0.015625f : 0.0f * a;
    const uint32_t cut = (__float_as_uint(a + low) + bits) & 0xfff00000u;
    return copysignf(__uint_as_float(cut) - low, v);
}

__device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x9e4a8af7u;
    h = (h ^ (h >> 15)) * 0xa6bd2c99u;
    return h ^ (h >> 16);
}

__device__ __forceinline__ float sqrt_approx(float v) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// The scale of a block whose largest magnitude in this lane is `top`, and 1 / scale.
// Below 2^-100 the block is zero: 448 / top would overflow.
__device__ __forceinline__ float2 block_scale(float top) {
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    if (top < 7.888609052210118e-31f) return make_float2(0.0f, 0.0f);
    return make_float2(top / 448.0f, 448.0f / top);
}

template <typename P, typename G, bool EIGHT, bool MASTER>
__device__ __forceinline__ void update(const Entry &e, const Rates &r, const Consts &k, uint32_t block) {
    const int lane = threadIdx.x & 31;
    const long long at = (long long)block * 256 + lane * 8;
    const int have = (int)max(0LL, min(8LL, e.numel - at));
    const bool full = have == 8;
    float p[8], g[8], m[8], v[8], root[8];
    load8<G>((const G *)e.grad + at, full, have, g);
    if (EIGHT) {
        load_e4m3((const uint8_t *)e.m + at, full, have, e.m_scale[block], m);
        load_e4m3((const uint8_t *)e.v + at, full, have, e.v_scale[block], v);
    } else {
        load8<float>((const float *)e.m + at, full, have, m);
        load8<float>((const float *)e.v + at, full, have, v);
    }
    if (MASTER)
        load8<float>(e.master + at, full, have, p);
    else
        load8<P>((const P *)e.param + at, full, have, p);
    float top_m = 0.0f, top_v = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        g[i] *= r.gs;
        if (EIGHT) v[i] *= v[i];
        m[i] = fmaf(k.b1, m[i], k.c1 * g[i]);
        v[i] = fmaf(k.b2, v[i], k.c2 * (g[i] * g[i]));
        root[i] = sqrt_approx(v[i]);
        const float den = fmaf(root[i], r.root_scale, k.eps);
        p[i] = fmaf(p[i], r.keep, -r.rate * __fdividef(m[i], den));
        if (EIGHT) {
            top_m = fmaxf(top_m, fabsf(m[i]));
            top_v = fmaxf(top_v, root[i]);
        }
    }
    if (MASTER) store8<float>(e.master + at, full, have, p);
    store8<P>((P *)e.param + at, full, have, p);
    if (!EIGHT) {
        store8<float>((float *)e.m + at, full, have, m);
        store8<float>((float *)e.v + at, full, have, v);
        return;
    }
    const float2 sm = block_scale(top_m), sv = block_scale(top_v);
    if (lane == 0) {
        e.m_scale[block] = sm.x;
        e.v_scale[block] = sv.x;
    }
    const uint32_t h0 = (uint32_t)at * 0x51f6db5bu + r.key;
    uint32_t wm[2], wv[2];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const uint32_t ha = mix(h0 + i * 0x51f6db5bu), hb = mix(h0 + (i + 1) * 0x51f6db5bu);
        const uint32_t two_m = e4m3x2(dither(m[i], sm.y, ((ha & 0xffffu) << 4) + 8), dither(m[i + 1], sm.y, ((hb & 0xffffu) << 4) + 8));
        const uint32_t two_v = e4m3x2(dither(root[i], sv.y, ((ha >> 16) << 4) + 8), dither(root[i + 1], sv.y, ((hb >> 16) << 4) + 8));
        if (i % 4 == 0) {
            wm[i >> 2] = two_m;
            wv[i >> 2] = two_v;
        } else {
            wm[i >> 2] |= two_m << 16;
            wv[i >> 2] |= two_v << 16;
        }
    }
    uint8_t *om = (uint8_t *)e.m + at, *ov = (uint8_t *)e.v + at;
    if (full) {
        *reinterpret_cast<uint2 *>(om) = make_uint2(wm[0], wm[1]);
        *reinterpret_cast<uint2 *>(ov) = make_uint2(wv[0], wv[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) {
                om[i] = (uint8_t)(wm[i >> 2] >> (8 * (i & 3)));
                ov[i] = (uint8_t)(wv[i >> 2] >> (8 * (i & 3)));
            }
    }
}

// Every warp walks blocks w, w + warps, ...; the tensor is found by bisection once and
// followed from there.
template <int MAX>
__global__ void __launch_bounds__(AT)
adamw_kernel(const __grid_constant__ Table<MAX> tab, const Consts k) {
    pdl_wait();
    const float gs = k.grad_scale ? *k.grad_scale : 1.0f;
    if (!isfinite(gs)) return;  // an overflowed gradient: the step is left out
    const int t = max(1, k.step + (k.step_dev ? *k.step_dev : 0));
    const float lr = k.lr * (k.lr_dev ? *k.lr_dev : 1.0f);
    const float inv_c1 = -1.0f / expm1f((float)t * k.log_b1), root_scale = 1.0f / sqrtf(-expm1f((float)t * k.log_b2));
    const uint32_t key = k.seed_key + (uint32_t)t * 0x339cd49bu;
    const uint32_t warps = gridDim.x * (AT / 32);
    uint32_t b = blockIdx.x * (AT / 32) + (threadIdx.x >> 5);
    int lo = 0, hi = tab.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tab.first[mid] <= b)
            lo = mid;
        else
            hi = mid;
    }
    for (; b < tab.blocks; b += warps) {
        while (lo + 1 < tab.n && tab.first[lo + 1] <= b) ++lo;
        const Entry &e = tab.e[lo];
        const float rate = lr * e.lr_scale;
        const Rates r = {1.0f - rate * e.decay, rate * inv_c1, root_scale, gs, key + e.key};
        const uint32_t block = b - tab.first[lo];
        switch (e.kind) {
            case P32 | G32: update<float, float, false, false>(e, r, k, block); break;
            case P32 | G32 | S8: update<float, float, true, false>(e, r, k, block); break;
            case 0: update<__nv_bfloat16, __nv_bfloat16, false, false>(e, r, k, block); break;
            case S8: update<__nv_bfloat16, __nv_bfloat16, true, false>(e, r, k, block); break;
            case MST: update<__nv_bfloat16, __nv_bfloat16, false, true>(e, r, k, block); break;
            case MST | S8: update<__nv_bfloat16, __nv_bfloat16, true, true>(e, r, k, block); break;
            case G32: update<__nv_bfloat16, float, false, false>(e, r, k, block); break;
            case G32 | S8: update<__nv_bfloat16, float, true, false>(e, r, k, block); break;
            case G32 | MST: update<__nv_bfloat16, float, false, true>(e, r, k, block); break;
            default: update<__nv_bfloat16, float, true, true>(e, r, k, block); break;  // G32 | S8 | MST
        }
    }
}

static_assert(sizeof(Table<380>) + sizeof(Consts) <= 32764, "a launch's arguments");

template <int MAX>
int launch_table(const vmoe_adamw_tensor *tensors, int n, int base, uint32_t blocks, const Consts &k, cudaStream_t s) {
    Table<MAX> tab;
    tab.n = 0;
    tab.blocks = blocks;
    uint32_t at = 0;
    for (int i = 0; i < n; ++i) {
        const vmoe_adamw_tensor &x = tensors[i];
        if (x.numel == 0) continue;
        Entry &e = tab.e[tab.n];
        tab.first[tab.n++] = at;
        at += (uint32_t)((x.numel + 255) / 256);
        e.param = x.param;
        e.grad = x.grad;
        e.m = x.m;
        e.v = x.v;
        e.m_scale = x.m_scale;
        e.v_scale = x.v_scale;
        e.master = x.master;
        e.numel = x.numel;
        e.lr_scale = x.lr_scale;
        e.decay = x.weight_decay;
        e.key = (uint32_t)(base + i) * 0x5e4087b3u;
        e.kind = (x.param_dtype == VMOE_F32 ? P32 : 0) | (x.grad_dtype == VMOE_F32 ? G32 : 0) |
                 (x.state == VMOE_STATE_E4M3 ? S8 : 0) | (x.master ? MST : 0);
    }
    const long long ctas = ((long long)blocks + AT / 32 - 1) / (AT / 32);
    return launch_kernel(adamw_kernel<MAX>, dim3((unsigned)std::min<long long>(ctas, 4LL * num_sms())), dim3(AT), 0, s, tab, k);
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
    k.step = c->step;
    k.seed_key = c->seed * 0xe32a5e87u;
    k.step_dev = c->step_dev;
    k.lr_dev = c->lr_dev;
    k.grad_scale = c->grad_scale;
    constexpr int SMALL = 40, LARGE = 380;  // tables of 3.4 and 32 KB; a launch takes at most 32764 B
    for (int base = 0; base < n;) {
        int m = 0;
        uint64_t blocks = 0;
        while (base + m < n && m < LARGE) {
            const uint64_t more = ((uint64_t)tensors[base + m].numel + 255) / 256;
            if (blocks + more > 0x7fffffffu) break;
            blocks += more;
            ++m;
        }
        if (blocks) {
            trace_before(s, "adamw");
            const int st = m <= SMALL ? launch_table<SMALL>(tensors + base, m, base, (uint32_t)blocks, k, s)
                                      : launch_table<LARGE>(tensors + base, m, base, (uint32_t)blocks, k, s);
            trace_after(s);
            if (st != VMOE_OK) return st;
        }
        base += m;
    }
    return VMOE_OK;
}

}  // namespace vmoe

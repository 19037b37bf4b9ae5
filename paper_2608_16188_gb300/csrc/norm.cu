// norm.cu -- what surrounds an expert layer in its transformer block (Section 2.1:
// the experts stand in the place of a ViT block's MLP): the norm behind the branch,
// its gate and the residual, and the norm ahead of the next layer, in one pass.
//
//   w = norm(y; post_w, post_b)      (or w = y)
//   z = rho x + gate . w             (rounded to the tokens' dtype as it is stored)
//   u = norm(z; pre_w, pre_b)        (of z as stored, so that the backward, which has
//                                     only that, differentiates what was computed)
// norm(v) = (v - mean) rstd . weight + bias, rstd = 1 / sqrt(var + eps); the root-mean-
// square form has mean = 0.  With dzt = dz + (d u / d z)^T du:
//   dx = rho dzt,   dy = (d w / d y)^T (gate . dzt),
//   A = sum_n dzt . yhat,  B = sum_n dzt,
//   dpost_w = gate . A,  dpost_b = gate . B,  dgate = post_w . A + post_b . B,
//   dpre_w = sum_n du . zhat,  dpre_b = sum_n du.
// gate and weights do not depend on the token, so two sums a column carry the three
// gradients behind the branch.  Variances are sums of squared distances to the mean
// (two passes over registers), all sums fp32.
#include <math.h>

#include <algorithm>

#include "common.cuh"

namespace vmoe {

namespace {

// Eight consecutive elements as they lie in memory, and as floats.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&o)[8]) const { bf16x8_to_f32(v, o); }
    // rounds in[] to what is stored
    __device__ __forceinline__ void set(float (&in)[8]) {
        v = f32_to_bf16x8(in);
        bf16x8_to_f32(v, in);
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = v; }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) {
        a = reinterpret_cast<const float4 *>(p)[0];
        b = reinterpret_cast<const float4 *>(p)[1];
    }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void get(float (&o)[8]) const {
        o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
        o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
    }
    __device__ __forceinline__ void set(float (&in)[8]) {
        a = make_float4(in[0], in[1], in[2], in[3]);
        b = make_float4(in[4], in[5], in[6], in[7]);
    }
    __device__ __forceinline__ void store(float *p) const {
        reinterpret_cast<float4 *>(p)[0] = a;
        reinterpret_cast<float4 *>(p)[1] = b;
    }
};

// Eight values of a [T, d] parameter, or a constant where there is none.
__device__ __forceinline__ void param8(const float *p, long long at, float none, float (&o)[8]) {
    if (p) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(p + at)), b = __ldg(reinterpret_cast<const float4 *>(p + at) + 1);
        o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
        o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = none;
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The sum over the W warps of a row, the same in every thread.
template <int W>
__device__ __forceinline__ float group_sum(float v, float *buf) {
    v = warp_sum(v);
    if (W == 1) return v;
    __syncthreads();  // the last sum's readers are done
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += buf[w];
    return v;
}

struct FwdArgs {
    const void *x, *y;
    const float *post_w, *post_b, *gate, *pre_w, *pre_b;
    void *z, *u;
    float2 *post_stat, *pre_stat;
    float eps, rho;
    bool rms, post;
};

// mean and rstd of the NV x 8 values a thread holds of a row.
template <int NV, int W>
__device__ __forceinline__ float2 stats(const float (&v)[NV][8], const bool (&have)[NV], int d, bool rms, float eps, float *buf) {
    float mean = 0.0f;
    if (!rms) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[j][i];
        mean = group_sum<W>(s, buf) / (float)d;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (!have[j]) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = v[j][i] - mean;
            q = fmaf(c, c, q);
        }
    }
    q = group_sum<W>(q, buf) / (float)d;
    return make_float2(mean, 1.0f / sqrtf(q + eps));
}

// Forward: W warps a row, NV vectors of 8 a thread.  With W = 1 the eight warps of a
// CTA take a row each.
template <typename T, int NV, int W>
__global__ void __launch_bounds__(W == 1 ? 256 : 32 * W)
norm_fwd_kernel(Dims p, FwdArgs a) {
    __shared__ float buf[32];
    constexpr int GROUPS = W == 1 ? 8 : 1, TH = 32 * W;
    const int th = threadIdx.x % TH, d = p.d;
    const long long row = (long long)blockIdx.x * GROUPS + threadIdx.x / TH;
    pdl_wait();
    if (row >= (long long)p.T * p.N) return;  // whole groups
    const long long par = row / p.N * d, at = row * d;
    float v[NV][8];
    bool have[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (th + j * TH) * 8;
        have[j] = c < d;
        Raw8<T> r;
        r.zero();
        if (have[j]) r.load((const T *)(a.y ? a.y : a.x) + at + c);
        r.get(v[j]);
    }
    if (a.y) {
        float2 s = make_float2(0.0f, 1.0f);
        if (a.post) {
            s = stats<NV, W>(v, have, d, a.rms, a.eps, buf);
            if (a.post_stat && th == 0) a.post_stat[row] = s;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!have[j]) continue;
            const int c = (th + j * TH) * 8;
            float x[8], g[8], w[8], b[8];
            Raw8<T> r;
            r.load((const T *)a.x + at + c);
            r.get(x);
            param8(a.gate, par + c, 1.0f, g);
            param8(a.post_w, par + c, 1.0f, w);
            param8(a.post_b, par + c, 0.0f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[j][i] = fmaf(g[i], fmaf((v[j][i] - s.x) * s.y, w[i], b[i]), a.rho * x[i]);
            r.set(v[j]);
            r.store((T *)a.z + at + c);
        }
    }
    if (!a.u) return;
    const float2 s = stats<NV, W>(v, have, d, a.rms, a.eps, buf);
    if (a.pre_stat && th == 0) a.pre_stat[row] = s;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (!have[j]) continue;
        const int c = (th + j * TH) * 8;
        float w[8], b[8];
        Raw8<T> r;
        param8(a.pre_w, par + c, 1.0f, w);
        param8(a.pre_b, par + c, 0.0f, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = fmaf((v[j][i] - s.x) * s.y, w[i], b[i]);
        r.set(v[j]);
        r.store((T *)a.u + at + c);
    }
}

// ---------------------------------------------------------------------------
// Backward.  W = ceil(d / 256) warps hold a row, 8 columns a thread; a CTA walks a
// slice of one task's rows with GROUPS such groups and keeps the four column sums in
// registers.  Its sums go to `parts` [T][slices][4][d]: A, B, dpre_w, dpre_b.
struct BwdArgs {
    const void *y, *z;
    const float2 *post_stat, *pre_stat;
    const float *post_w, *post_b, *gate, *pre_w;
    const void *dz, *du;
    void *dx, *dy;
    float *parts;
    float rho;
    bool rms, post;
};

int bwd_warps(int d) { return (d + 255) / 256; }
int bwd_groups(int d) { return std::max(1, 8 / bwd_warps(d)); }
int bwd_slices(const Dims &p) {
    const int rows = 4 * bwd_groups(p.d);
    return std::max(1, std::min((p.N + rows - 1) / rows, (456 + p.T - 1) / p.T));  // 152 SMs x 3
}

// Sums of two values over the warps of each group.
__device__ __forceinline__ float2 rows_sum(float a, float b, int W, int group, float2 *buf) {
    a = warp_sum(a);
    b = warp_sum(b);
    if (W == 1) return make_float2(a, b);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = make_float2(0.0f, 0.0f);
    for (int w = 0; w < W; ++w) {
        const float2 o = buf[group * W + w];
        s.x += o.x;
        s.y += o.y;
    }
    return s;
}

template <typename T, int MAXT>
__global__ void __launch_bounds__(MAXT)
norm_bwd_kernel(Dims p, BwdArgs a, int W, int groups) {
    __shared__ float2 buf[32];
    extern __shared__ float join[];  // [groups - 1][4][d], where there are several groups
    const int th = threadIdx.x % (32 * W), group = threadIdx.x / (32 * W);
    const int t = blockIdx.y, N = p.N, d = p.d, c = 8 * th;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    const bool have = c < d;
    const float share = 1.0f / (float)d, centre = a.rms ? 0.0f : share;
    pdl_wait();
    float pw[8], aw[8];  // pre_w; gate . post_w
    {
        const long long par = (long long)t * d + c;
        float g[8];
        param8(have ? a.pre_w : nullptr, par, 1.0f, pw);
        param8(have ? a.gate : nullptr, par, 1.0f, g);
        param8(have ? a.post_w : nullptr, par, 1.0f, aw);
#pragma unroll
        for (int i = 0; i < 8; ++i) aw[i] *= g[i];
    }
    float A[8] = {}, B[8] = {}, Pw[8] = {}, Pb[8] = {};
    for (int n0 = beg; n0 < end; n0 += groups) {
        const int n = n0 + group;
        const bool in = have && n < end;
        const long long row = (long long)t * N + min(n, end - 1), at = row * d + c;
        Raw8<T> ry, rz, rdz, rdu;
        ry.zero();
        rz.zero();
        rdz.zero();
        rdu.zero();
        if (in) {
            if (a.dz) rdz.load((const T *)a.dz + at);
            if (a.du) {
                rdu.load((const T *)a.du + at);
                rz.load((const T *)a.z + at);
            }
            if (a.y) ry.load((const T *)a.y + at);
        }
        float dz[8];
        rdz.get(dz);
        if (a.du) {
            const float2 s = a.pre_stat[row];
            float zh[8], du[8];
            rz.get(zh);
            rdu.get(du);
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                zh[i] = in ? (zh[i] - s.x) * s.y : 0.0f;
                Pw[i] = fmaf(du[i], zh[i], Pw[i]);
                Pb[i] += du[i];
                du[i] *= pw[i];
                s1 += du[i];
                s2 = fmaf(du[i], zh[i], s2);
            }
            const float2 q = rows_sum(s1, s2, W, group, buf);
            const float m1 = q.x * centre, m2 = q.y * share;
#pragma unroll
            for (int i = 0; i < 8; ++i) dz[i] = fmaf(s.y, (du[i] - m1) - zh[i] * m2, dz[i]);
        }
        if (a.y) {
            const float2 s = a.post ? a.post_stat[row] : make_float2(0.0f, 1.0f);
            float yh[8], g[8], s1 = 0.0f, s2 = 0.0f;
            ry.get(yh);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!in) dz[i] = 0.0f;
                yh[i] = in ? (yh[i] - s.x) * s.y : 0.0f;
                A[i] = fmaf(dz[i], yh[i], A[i]);
                B[i] += dz[i];
                g[i] = dz[i] * aw[i];
                s1 += g[i];
                s2 = fmaf(g[i], yh[i], s2);
            }
            if (a.post) {
                const float2 q = rows_sum(s1, s2, W, group, buf);
                const float m1 = q.x * centre, m2 = q.y * share;
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = s.y * ((g[i] - m1) - yh[i] * m2);
            }
            if (in) {
                Raw8<T> r;
                r.set(g);
                r.store((T *)a.dy + at);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) dz[i] *= a.rho;
        }
        if (in) {
            Raw8<T> r;
            r.set(dz);
            r.store((T *)a.dx + at);
        }
    }
    // the groups' sums, in their order
    __syncthreads();
    if (group > 0 && have) {
        float *o = join + (long long)(group - 1) * 4 * d + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            o[i] = A[i];
            o[d + i] = B[i];
            o[2 * d + i] = Pw[i];
            o[3 * d + i] = Pb[i];
        }
    }
    __syncthreads();
    if (group > 0 || !have) return;
    for (int g = 1; g < groups; ++g) {
        const float *o = join + (long long)(g - 1) * 4 * d + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            A[i] += o[i];
            B[i] += o[d + i];
            Pw[i] += o[2 * d + i];
            Pb[i] += o[3 * d + i];
        }
    }
    float *o = a.parts + ((long long)t * gridDim.x + blockIdx.x) * 4 * d + c;
    Raw8<float> r;
    r.set(A);
    r.store(o);
    r.set(B);
    r.store(o + d);
    r.set(Pw);
    r.store(o + 2 * d);
    r.set(Pb);
    r.store(o + 3 * d);
}

struct JoinArgs {
    const float *parts, *post_w, *post_b, *gate;
    float *dpost_w, *dpost_b, *dgate, *dpre_w, *dpre_b;
};

// The slices' column sums joined: 32 columns a CTA, eight threads a column, each a run
// of the slices.
__global__ void __launch_bounds__(256)
norm_join_kernel(Dims p, JoinArgs a, int slices) {
    __shared__ float part[8][4][32];
    const int lane = threadIdx.x & 31, q = threadIdx.x >> 5, d = p.d, t = blockIdx.y, c = blockIdx.x * 32 + lane;
    const int beg = slices * q / 8, end = slices * (q + 1) / 8;
    pdl_wait();
    float s[4] = {};
    if (c < d)
        for (int i = beg; i < end; ++i) {
            const float *in = a.parts + ((long long)t * slices + i) * 4 * d + c;
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += in[(long long)j * d];
        }
#pragma unroll
    for (int j = 0; j < 4; ++j) part[q][j][lane] = s[j];
    __syncthreads();
    if (q > 0 || c >= d) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[j] += part[i][j][lane];
    }
    const long long at = (long long)t * d + c;
    const float g = a.gate ? a.gate[at] : 1.0f, w = a.post_w ? a.post_w[at] : 1.0f, b = a.post_b ? a.post_b[at] : 0.0f;
    if (a.dpost_w) a.dpost_w[at] = g * s[0];
    if (a.dpost_b) a.dpost_b[at] = g * s[1];
    if (a.dgate) a.dgate[at] = fmaf(w, s[0], b * s[1]);
    if (a.dpre_w) a.dpre_w[at] = s[2];
    if (a.dpre_b) a.dpre_b[at] = s[3];
}

template <typename T, int NV, int W>
int launch_fwd(const Dims &p, const FwdArgs &a, cudaStream_t s) {
    const long long rows = (long long)p.T * p.N, groups = W == 1 ? 8 : 1;
    return launch_kernel(norm_fwd_kernel<T, NV, W>, dim3((unsigned)((rows + groups - 1) / groups)), dim3(W == 1 ? 256 : 32 * W),
                         0, s, p, a);
}
template <typename T>
int run_fwd(const Dims &p, const FwdArgs &a, cudaStream_t s) {
    if (p.d <= 256) return launch_fwd<T, 1, 1>(p, a, s);
    if (p.d <= 512) return launch_fwd<T, 2, 1>(p, a, s);
    if (p.d <= 768) return launch_fwd<T, 3, 1>(p, a, s);
    if (p.d <= 1024) return launch_fwd<T, 4, 1>(p, a, s);
    if (p.d <= 2048) return launch_fwd<T, 4, 2>(p, a, s);
    if (p.d <= 4096) return launch_fwd<T, 4, 4>(p, a, s);
    return launch_fwd<T, 4, 8>(p, a, s);
}

template <typename T>
int run_bwd(const Dims &p, const BwdArgs &a, cudaStream_t s) {
    const int W = bwd_warps(p.d), groups = bwd_groups(p.d), threads = 32 * W * groups;
    const size_t smem = (size_t)(groups - 1) * 4 * p.d * sizeof(float);
    const dim3 grid(bwd_slices(p), p.T);
    if (threads <= 256) return launch_kernel(norm_bwd_kernel<T, 256>, grid, dim3(threads), smem, s, p, a, W, groups);
    return launch_kernel(norm_bwd_kernel<T, 1024>, grid, dim3(threads), smem, s, p, a, W, groups);
}

}  // namespace

size_t norm_bwd_workspace(const Dims &p) { return (size_t)p.T * bwd_slices(p) * 4 * p.d * sizeof(float); }

int launch_block_norm(const Dims &p, const vmoe_norm *n, const void *x, const void *y, const float *post_w,
                      const float *post_b, const float *gate, const float *pre_w, const float *pre_b, void *z, void *u,
                      float *post_stat, float *pre_stat, cudaStream_t s) {
    const FwdArgs a = {x, y, post_w, post_b, gate, pre_w, pre_b, z, u, (float2 *)post_stat, (float2 *)pre_stat,
                       n->eps, n->residual_scale, (n->flags & VMOE_NORM_RMS) != 0, (n->flags & VMOE_NORM_POST) != 0};
    trace_before(s, "block_norm");
    const int st = p.bf16 ? run_fwd<__nv_bfloat16>(p, a, s) : run_fwd<float>(p, a, s);
    trace_after(s);
    return st;
}

int launch_block_norm_bwd(const Dims &p, const vmoe_norm *n, const void *y, const void *z, const float *post_stat,
                          const float *pre_stat, const float *post_w, const float *post_b, const float *gate,
                          const float *pre_w, const void *dz, const void *du, void *dx, void *dy, float *dpost_w,
                          float *dpost_b, float *dgate, float *dpre_w, float *dpre_b, float *parts, cudaStream_t s) {
    const BwdArgs a = {y, z, (const float2 *)post_stat, (const float2 *)pre_stat, post_w, post_b, gate, pre_w, dz, du,
                       dx, dy, parts, n->residual_scale, (n->flags & VMOE_NORM_RMS) != 0, (n->flags & VMOE_NORM_POST) != 0};
    trace_before(s, "block_norm_bwd");
    int st = p.bf16 ? run_bwd<__nv_bfloat16>(p, a, s) : run_bwd<float>(p, a, s);
    trace_after(s);
    if (st != VMOE_OK || !(dpost_w || dpost_b || dgate || dpre_w || dpre_b)) return st;
    const JoinArgs j = {parts, post_w, post_b, gate, dpost_w, dpost_b, dgate, dpre_w, dpre_b};
    trace_before(s, "block_norm_join");
    st = launch_kernel(norm_join_kernel, dim3((p.d + 31) / 32, p.T), dim3(256), 0, s, p, j, bwd_slices(p));
    trace_after(s);
    return st;
}

}  // namespace vmoe

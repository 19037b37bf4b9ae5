// head.cu -- the losses behind the blocks (Section 3.1 adapts the visual module and its projector; the tasks' answers are
// entries of a vocabulary, and the devices' models are taught by a larger one): softmax cross entropy over a large
// vocabulary and distillation from a teacher's largest logits, with their gradients, without keeping the logits.
//
//   l = z w^T;  ce = lse(l) - l_y;  kl = sum_j q_j (log q_j - log p_{i_j}),  p the softmax of l / tau, q that of the
//   teacher's entries / tau
//   dl = (dce + dlse) softmax(l) - dce 1[y] + dkl / tau (p - q);  dz = dl w;  dw = dl^T z
//
// What bounds it: the products, 2 N V d operations each: one forward, two for the gradients, and the logits once more,
// which are not kept: dl is formed in bf16 for a piece of the vocabulary at a time (head_tc.cu).  A step is four products
// where the least is three.
//
// Only tokens that take part are multiplied: head_rows packs their numbers, head_gather copies their rows (fp32 ones
// as three bf16 parts), so padding and prompts cost nothing, and what lies in them is not looked at.
#include <math.h>

#include <algorithm>

#include "head.cuh"

namespace vmoe {
namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr float LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;
constexpr int HR_THREADS = 1024, HG_THREADS = 256, HF_ROWS = 32;

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

struct Sizes {
    int T, N, Np, d, V, K;
};

__device__ __forceinline__ bool entry_ok(const Sizes &z, int i, float l) { return i >= 0 && i < z.V && l != -INFINITY; }
__device__ __forceinline__ bool label_ok(const Sizes &z, int y) { return y >= 0 && y < z.V; }
__device__ __forceinline__ bool taught(const Sizes &z, const int32_t *tidx, const float *tlogit, long long tn) {
    for (int j = 0; j < z.K; ++j)
        if (entry_ok(z, tidx[tn * z.K + j], tlogit[tn * z.K + j])) return true;  // the first, as a rule
    return false;
}

// The tokens of a head that take part, in order: map[row] = token, pos[token] = row or -1.  A CTA a head.
__global__ void __launch_bounds__(HR_THREADS)
head_rows_kernel(Sizes z, const int32_t *__restrict__ label, const int32_t *__restrict__ tidx,
                 const float *__restrict__ tlogit, int *__restrict__ rows, int *__restrict__ pos, int *__restrict__ map) {
    __shared__ int sums[32], total;
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    int run = 0;
    for (int n0 = 0; n0 < z.N; n0 += HR_THREADS) {
        const int n = n0 + tid;
        const long long tn = (long long)t * z.N + n;
        bool in = false;
        if (n < z.N) in = (label && label_ok(z, label[tn])) || (tidx && taught(z, tidx, tlogit, tn));
        const unsigned mask = __ballot_sync(FULL, in);
        if (lane == 0) sums[warp] = __popc(mask);
        __syncthreads();
        if (warp == 0) {
            const int c = sums[lane];
            int incl = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(FULL, incl, o);
                if (lane >= o) incl += y;
            }
            sums[lane] = incl - c;
            if (lane == 31) total = incl;
        }
        __syncthreads();
        const int r = run + sums[warp] + __popc(mask & ((1u << lane) - 1u));
        if (n < z.N) pos[tn] = in ? r : -1;
        if (in) map[(long long)t * z.Np + r] = n;
        run += total;
        __syncthreads();
    }
    if (tid == 0) rows[t] = run;
}

// Their tokens' rows, packed; the rest of the last tile is zeros.  A warp a row.
template <typename T>
__global__ void __launch_bounds__(HG_THREADS)
head_gather_kernel(Sizes z, const T *__restrict__ src, const int32_t *__restrict__ label, const int *__restrict__ rows,
                   const int *__restrict__ map, int *__restrict__ out_label, __nv_bfloat16 *__restrict__ out) {
    const int t = blockIdx.y, lane = threadIdx.x & 31, r = blockIdx.x * (HG_THREADS / 32) + (threadIdx.x >> 5);
    pdl_wait();
    const int n = rows[t];
    if (r >= (n + HEAD_TILE - 1) / HEAD_TILE * HEAD_TILE) return;
    const long long at = (long long)t * z.Np + r, tn = r < n ? (long long)t * z.N + map[at] : 0;
    if (out_label && lane == 0) out_label[at] = r < n && label_ok(z, label[tn]) ? label[tn] : -1;
    const long long plane = (long long)z.T * z.Np * z.d;
    for (int c = lane * 8; c < z.d; c += 256) {
        if constexpr (sizeof(T) == 2) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < n) v = __ldg(reinterpret_cast<const uint4 *>(src + tn * z.d + c));
            *reinterpret_cast<uint4 *>(out + at * z.d + c) = v;
        } else {
            __align__(16) __nv_bfloat16 p[3][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) split3(r < n ? __ldg(src + tn * z.d + c + i) : 0.0f, p[0][i], p[1][i], p[2][i]);
#pragma unroll
            for (int i = 0; i < 3; ++i)
                *reinterpret_cast<uint4 *>(out + i * plane + at * z.d + c) = *reinterpret_cast<const uint4 *>(p[i]);
        }
    }
}

// fp32 weights as three bf16 parts.  n: a multiple of 8.
__global__ void __launch_bounds__(HG_THREADS)
head_split_kernel(long long n, const float *__restrict__ src, __nv_bfloat16 *__restrict__ out) {
    pdl_wait();
    for (long long i = ((long long)blockIdx.x * HG_THREADS + threadIdx.x) * 8; i < n; i += (long long)gridDim.x * HG_THREADS * 8) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(src + i)), b = __ldg(reinterpret_cast<const float4 *>(src + i) + 1);
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        __align__(16) __nv_bfloat16 p[3][8];
#pragma unroll
        for (int q = 0; q < 8; ++q) split3(v[q], p[0][q], p[1][q], p[2][q]);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(out + q * n + i) = *reinterpret_cast<const uint4 *>(p[q]);
    }
}

template <typename T>
__device__ __forceinline__ void load8(const T *p, float *o);
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16 *p, float *o) {
    bf16x8_to_f32(__ldg(reinterpret_cast<const uint4 *>(p)), o);
}
template <>
__device__ __forceinline__ void load8<float>(const float *p, float *o) {
    const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
    o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
}

// A teacher's distribution over a token's entries: lane l has entries l, l + 32, ...  lq: log q (natural).
struct Teacher {
    static constexpr int M = HEAD_K / 32;
    int i[M];
    float q[M], lq[M];
    bool any;
    __device__ __forceinline__ void load(const Sizes &z, const int32_t *tidx, const float *tlogit, float inv_tau, long long tn) {
        const int lane = threadIdx.x & 31;
        float t[M], top = -INFINITY;
        bool here = false;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int j = lane + 32 * m;
            i[m] = j < z.K ? tidx[tn * z.K + j] : -1;
            t[m] = j < z.K ? tlogit[tn * z.K + j] : -INFINITY;
            if (!entry_ok(z, i[m], t[m])) i[m] = -1;
            if (i[m] < 0) continue;
            t[m] *= inv_tau;
            top = fmaxf(top, t[m]);
            here = true;
        }
        any = __any_sync(FULL, here);
        top = warp_max(top);
        float sum = 0.0f;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            q[m] = i[m] >= 0 ? expf(t[m] - top) : 0.0f;
            sum += q[m];
        }
        sum = warp_sum(sum);
        const float ls = logf(sum);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            q[m] = i[m] >= 0 ? q[m] / sum : 0.0f;
            lq[m] = i[m] >= 0 ? t[m] - top - ls : 0.0f;
        }
    }
};

// The losses from the tiles' sums, 32 packed rows a CTA: each warp joins every eighth half tile of all rows, the first
// warp the warps' sums; then, with a teacher, a warp a row: the logits of its entries, each a dot product.
// CTAs past the last row leave zeros at the tokens without a part.
struct Finish {
    Sizes z;
    int halves, pitch;  // half tiles of the vocabulary, and as the sums are laid out
    int stats;
    float inv_tau, c1;
    const int *rows, *pos, *map, *label;
    const float2 *part, *part2;
    const float *picked;
    const int32_t *tidx;
    const float *tlogit;
    float *ce, *lse, *kl, *tlse, *logp;
};
__device__ __forceinline__ void join(float &m, float &s, float2 v) {
    const float top = fmaxf(m, v.x);
    s = s * exp2f(m - top) + v.y * exp2f(v.x - top);
    m = top;
}
template <typename T>
__global__ void __launch_bounds__(HG_THREADS)
head_finish_kernel(Finish f, const T *__restrict__ zt, const T *__restrict__ w) {
    __shared__ float2 sm[2][HG_THREADS / 32][32];
    __shared__ float tl[32];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Sizes z = f.z;
    pdl_wait();
    // tokens without a part
    for (int n = blockIdx.x * HG_THREADS + tid; n < z.N; n += gridDim.x * HG_THREADS) {
        const long long tn = (long long)t * z.N + n;
        if (f.pos[tn] >= 0) continue;
        if (f.ce) f.ce[tn] = f.lse[tn] = 0.0f;
        if (f.kl) {
            f.kl[tn] = f.tlse[tn] = 0.0f;
            for (int j = 0; j < z.K; ++j) f.logp[tn * z.K + j] = 0.0f;
        }
    }
    const int n = f.rows[t], r0 = blockIdx.x * HF_ROWS;
    if (r0 >= n) return;
    float m = -INFINITY, s = 0.0f, m2 = -INFINITY, s2 = 0.0f;
    const float2 *p = f.part + (long long)t * f.pitch * z.Np + r0 + lane;
    const float2 *p2 = f.stats == 2 ? f.part2 + (long long)t * f.pitch * z.Np + r0 + lane : nullptr;
#pragma unroll 4
    for (int h = warp; h < f.halves; h += HG_THREADS / 32) {
        join(m, s, p[(long long)h * z.Np]);
        if (p2) join(m2, s2, p2[(long long)h * z.Np]);
    }
    sm[0][warp][lane] = make_float2(m, s);
    sm[1][warp][lane] = make_float2(m2, s2);
    __syncthreads();
    const int row = r0 + lane;
    if (warp == 0) {
        for (int q = 1; q < HG_THREADS / 32; ++q) {
            join(m, s, sm[0][q][lane]);
            if (p2) join(m2, s2, sm[1][q][lane]);
        }
        const float ls = log2f(s), a = (m + ls) * LN2, b = p2 ? (m2 + log2f(s2)) * LN2 : a;
        tl[lane] = b;
        if (row < n && f.ce) {
            const long long at = (long long)t * z.Np + row, tn = (long long)t * z.N + f.map[at];
            const bool has = f.label[at] >= 0;
            f.ce[tn] = has ? ((m - f.picked[at] * f.c1) + ls) * LN2 : 0.0f;  // a sure token's is small: no difference of large ones
            f.lse[tn] = has ? a : 0.0f;
        }
    }
    if (!f.kl) return;
    __syncthreads();
    for (int i = warp; i < HF_ROWS && r0 + i < n; i += HG_THREADS / 32) {
        const long long tn = (long long)t * z.N + f.map[(long long)t * z.Np + r0 + i];
        Teacher q;
        q.load(z, f.tidx, f.tlogit, f.inv_tau, tn);
        const T *zr = zt + tn * z.d, *wt = w + (long long)t * z.V * z.d;
        float loss = 0.0f;
#pragma unroll
        for (int mm = 0; mm < Teacher::M; ++mm) {
            if (32 * mm >= z.K) break;
            float mine = 0.0f;  // lane l: entry 32 mm + l
            const int last = min(32, z.K - 32 * mm);
            for (int j = 0; j < last; j += 4) {  // four entries' rows at a time
                float acc[4] = {};
                const T *wr[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) wr[e] = wt + (long long)max(0, __shfl_sync(FULL, q.i[mm], (j + e) & 31)) * z.d;
                for (int c = lane * 8; c < z.d; c += 256) {
                    float a[8];
                    load8<T>(zr + c, a);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float b[8];
                        load8<T>(wr[e] + c, b);
#pragma unroll
                        for (int x = 0; x < 8; ++x) acc[e] = fmaf(a[x], b[x], acc[e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[e] = warp_sum(acc[e]);
                    if (lane == j + e) mine = acc[e];
                }
            }
            const float lp = q.i[mm] >= 0 ? mine * f.inv_tau - tl[i] : 0.0f;
            if (lane + 32 * mm < z.K) f.logp[tn * z.K + lane + 32 * mm] = lp;
            // an entry of no weight adds nothing, whatever its logarithm
            if (q.q[mm] > 0.0f || q.q[mm] != q.q[mm]) loss += q.q[mm] * (q.lq[mm] - lp);
        }
        loss = warp_sum(loss);
        if (lane == 0) {
            f.kl[tn] = q.any ? loss : 0.0f;
            f.tlse[tn] = q.any ? tl[i] : 0.0f;
        }
    }
}

// What HEAD_DLOGITS takes each row's exponentials times, and off at the label.  A thread a packed row.
struct Coef {
    Sizes z;
    float inv_tau;
    bool one;  // labels and a teacher at temperature 1: one exponential for both
    const int *rows, *map;
    const int32_t *label, *tidx;
    const float *tlogit, *ce, *lse, *tlse, *dce, *dlse, *dkl;
    float4 *coef;
    float *at_label;
};
// At the label dce (p - 1) + dlse p with p = exp(-ce): ce is kept to 2^-24 of itself or of 1, p and 1 would cancel.
__device__ __forceinline__ float label_value(float ce, float dce, float dlse) { return dce * expm1f(-ce) + dlse * expf(-ce); }
__global__ void __launch_bounds__(HG_THREADS) head_coef_kernel(Coef f) {
    const int t = blockIdx.y, r = blockIdx.x * HG_THREADS + threadIdx.x;
    pdl_wait();
    if (r >= f.rows[t]) return;
    const long long at = (long long)t * f.z.Np + r, tn = (long long)t * f.z.N + f.map[at];
    float4 c = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float there = 0.0f;
    const bool has = f.label && label_ok(f.z, f.label[tn]);
    if (has) {
        const float dce = f.dce ? f.dce[tn] : 0.0f, dlse = f.dlse ? f.dlse[tn] : 0.0f;
        there = label_value(f.ce[tn], dce, dlse);
        c.x = dce + dlse;
        c.y = f.lse[tn] * LOG2E;
    }
    if (f.tidx && f.dkl && taught(f.z, f.tidx, f.tlogit, tn)) {
        const float b = f.dkl[tn] * f.inv_tau;
        if (f.one) {
            c.x += b;
            c.y = f.tlse[tn] * LOG2E;
            if (has) there += b * expf(-f.ce[tn]);
        } else {
            c.z = b;
            c.w = f.tlse[tn] * LOG2E;
        }
    }
    f.coef[at] = c;
    f.at_label[at] = there;
}

// The teacher's entries in a piece of dl: the whole value, from the stored logarithms, so that neither the order of
// equal entries nor a label among them matters.  A warp a packed row.
struct Patch {
    Sizes z;
    int v0, vn, piece, parts;
    float tau, inv_tau;
    const int *rows, *map;
    const int32_t *label, *tidx;
    const float *tlogit, *ce, *lse, *tlse, *logp, *dce, *dlse, *dkl;
    __nv_bfloat16 *dl;
};
__global__ void __launch_bounds__(HG_THREADS) head_patch_kernel(Patch f) {
    const int t = blockIdx.y, lane = threadIdx.x & 31, r = blockIdx.x * (HG_THREADS / 32) + (threadIdx.x >> 5);
    const Sizes z = f.z;
    pdl_wait();
    if (r >= f.rows[t]) return;
    const long long at = (long long)t * z.Np + r, tn = (long long)t * z.N + f.map[at];
    Teacher q;
    q.load(z, f.tidx, f.tlogit, f.inv_tau, tn);
    if (!q.any) return;
    const int y = f.label && label_ok(z, f.label[tn]) ? f.label[tn] : -1;
    const float dce = y >= 0 && f.dce ? f.dce[tn] : 0.0f, dlse = y >= 0 && f.dlse ? f.dlse[tn] : 0.0f;
    const float b = f.dkl[tn] * f.inv_tau, lse = y >= 0 ? f.lse[tn] : 0.0f, tlse = f.tlse[tn];
    const long long plane = (long long)z.T * z.Np * f.piece;
    __nv_bfloat16 *row = f.dl + at * f.piece;
#pragma unroll
    for (int m = 0; m < Teacher::M; ++m) {
        if (32 * m >= z.K) break;
        const int i = q.i[m];
        float all = 0.0f;  // q of every entry with this index
#pragma unroll
        for (int o = 0; o < Teacher::M; ++o) {
            if (32 * o >= z.K) break;
            for (int j = 0; j < 32; ++j) {
                const int oi = __shfl_sync(FULL, q.i[o], j);
                const float oq = __shfl_sync(FULL, q.q[o], j);
                if (oi == i) all += oq;
            }
        }
        if (i < f.v0 || i >= f.v0 + f.vn) continue;
        const float lp = f.logp[tn * z.K + lane + 32 * m];
        float v = b * (expf(lp) - all);
        if (y >= 0) v += i == y ? label_value(f.ce[tn], dce, dlse) : (dce + dlse) * expf(f.tau * (lp + tlse) - lse);
        __nv_bfloat16 *o = row + (i - f.v0);
        if (f.parts == 1) {
            *o = __float2bfloat16_rn(v);
        } else {
            split3(v, o[0], o[plane], o[2 * plane]);
        }
    }
}

// dz from the parts of the sum; 0 for a token without a part.  Eight columns a thread.
template <typename T>
__global__ void __launch_bounds__(HG_THREADS)
head_dz_kernel(Sizes z, int splits, const int *__restrict__ pos, const float *__restrict__ parts, T *__restrict__ dz) {
    pdl_wait();
    const int vec = z.d / 8;
    const long long total = (long long)z.T * z.N * vec, plane = (long long)z.T * z.Np * z.d;
    for (long long i = (long long)blockIdx.x * HG_THREADS + threadIdx.x; i < total; i += (long long)gridDim.x * HG_THREADS) {
        const long long tn = i / vec;
        const int c = (int)(i - tn * vec) * 8, r = pos[tn];
        float v[8] = {};
        if (r >= 0) {
            const float *src = parts + ((tn / z.N) * z.Np + r) * z.d + c;
            for (int s = 0; s < splits; ++s) {
                float o[8];
                load8<float>(src + s * plane, o);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] += o[q];
            }
        }
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(dz + tn * z.d + c) = f32_to_bf16x8(v);
        } else {
            reinterpret_cast<float4 *>(dz + tn * z.d + c)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(dz + tn * z.d + c)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
}

Sizes sizes_of(const HeadPlan &h) { return Sizes{h.T, h.N, h.Np, h.d, h.V, h.K}; }
template <typename P>
P *at(void *ws, size_t offset) {
    return reinterpret_cast<P *>(static_cast<uint8_t *>(ws) + offset);
}

// Packed rows and, in fp32, the weights' parts: what both directions begin with.
int prepare(const Dims &p, const HeadPlan &h, const HeadIn &in, void *ws, const __nv_bfloat16 **zp, const __nv_bfloat16 **wp,
            cudaStream_t s) {
    const Sizes z = sizes_of(h);
    int *rows = at<int>(ws, h.rows), *pos = at<int>(ws, h.pos), *map = at<int>(ws, h.map), *label = at<int>(ws, h.label);
    __nv_bfloat16 *zc = at<__nv_bfloat16>(ws, h.z);
    trace_before(s, "head_rows");
    int st = launch_kernel(head_rows_kernel, dim3(h.T), dim3(HR_THREADS), 0, s, z, in.label, in.tidx, in.tlogit, rows, pos, map);
    trace_after(s);
    if (st != VMOE_OK) return st;
    trace_before(s, "head_gather");
    const dim3 grid(h.Np / (HG_THREADS / 32), h.T);
    int *lab = in.label ? label : nullptr;
    st = p.bf16 ? launch_kernel(head_gather_kernel<__nv_bfloat16>, grid, dim3(HG_THREADS), 0, s, z, (const __nv_bfloat16 *)in.z,
                                in.label, rows, map, lab, zc)
                : launch_kernel(head_gather_kernel<float>, grid, dim3(HG_THREADS), 0, s, z, (const float *)in.z, in.label, rows,
                                map, lab, zc);
    trace_after(s);
    if (st != VMOE_OK) return st;
    *zp = zc;
    *wp = (const __nv_bfloat16 *)in.w;
    if (!p.bf16) {
        __nv_bfloat16 *ws3 = at<__nv_bfloat16>(ws, h.w);
        const long long n = (long long)h.T * h.V * h.d, blocks = (n / 8 + HG_THREADS - 1) / HG_THREADS;
        trace_before(s, "head_split");
        st = launch_kernel(head_split_kernel, dim3((unsigned)std::min(blocks, 16LL * num_sms())), dim3(HG_THREADS), 0, s, n,
                           (const float *)in.w, ws3);
        trace_after(s);
        *wp = ws3;
    }
    return st;
}

}  // namespace

bool head_plan(const Dims &p, const vmoe_head *head, bool label, size_t bytes, HeadPlan *out) {
    HeadPlan h = {};
    const bool shared = (head->flags & VMOE_HEAD_SHARED) != 0;
    h.T = shared ? 1 : p.T;
    h.N = shared ? p.T * p.N : p.N;
    h.d = p.d;
    h.V = head->V;
    h.K = head->teacher_k;
    h.Np = (h.N + HEAD_TILE - 1) / HEAD_TILE * HEAD_TILE;
    h.parts = p.bf16 ? 1 : 3;
    h.tau = head->temperature;
    h.stats = label && h.K > 0 && head->temperature != 1.0f ? 2 : 1;
    h.c2 = (float)(1.4426950408889634 / (double)head->temperature);
    h.c1 = h.stats == 1 && h.K > 0 ? h.c2 : LOG2E;
    const size_t rowsp = (size_t)h.T * h.Np, tiles_v = ((size_t)h.V + HEAD_TILE - 1) / HEAD_TILE;
    size_t o = 0;
    auto take = [&](size_t n) {
        const size_t a = o;
        o += (n + 255) & ~(size_t)255;
        return a;
    };
    h.rows = take((size_t)h.T * 4);
    h.pos = take((size_t)h.T * h.N * 4);
    h.map = take(rowsp * 4);
    h.label = take(rowsp * 4);
    h.z = take(rowsp * h.d * 2 * h.parts);
    h.w = take(p.bf16 ? 0 : (size_t)h.T * h.V * h.d * 6);
    const size_t both = o;
    h.part = take(rowsp * tiles_v * 2 * 8);
    h.part2 = take(h.K > 0 ? rowsp * tiles_v * 2 * 8 : 0);
    h.picked = take(rowsp * 4);
    const size_t fwd = o;
    o = both;
    h.coef = take(rowsp * 16);
    h.at_label = take(rowsp * 4);
    // parts of dz's sum: while its tiles do not fill the SM pairs twice and each keeps 16 blocks of 64
    const size_t tiles_dz = (rowsp / HEAD_TILE) * ((h.d + HEAD_TILE - 1) / HEAD_TILE), pairs = num_sms() / 2;
    size_t splits = 1;
    while (splits < 16 && tiles_dz * splits * 2 <= pairs * 2 && tiles_v * 4 >= splits * 2 * 16) splits *= 2;
    const size_t fixed = o, column = rowsp * HEAD_TILE * 2 * h.parts;  // a tile of columns of dl
    size_t cols = tiles_v;
    const size_t want = (size_t)2 << 30;
    if (bytes == 0) {
        if (cols * column > want) cols = std::max<size_t>(1, want / column);
    } else {
        if (bytes < fwd) return false;
        auto rest = [&](size_t sp) {
            const size_t dzp = (sp * rowsp * h.d * 4 + 255) & ~(size_t)255;
            return bytes < fixed + dzp ? 0 : (bytes - fixed - dzp) / column;
        };
        while (splits > 1 && rest(splits) < 1) splits /= 2;
        cols = std::min(cols, rest(splits));
        if (cols < 1) return false;
    }
    h.splits = (int)splits;
    h.piece = (int)(cols * HEAD_TILE);
    h.dl = take(cols * column);
    h.dzp = take(splits * rowsp * h.d * 4);
    h.bytes = std::max(o, fwd);
    *out = h;
    return true;
}

size_t head_min_workspace(const Dims &p, const vmoe_head *head) {
    HeadPlan h;
    if (!head_plan(p, head, true, 0, &h)) return 0;
    const size_t rowsp = (size_t)h.T * h.Np, dzp = (rowsp * h.d * 4 + 255) & ~(size_t)255;
    const size_t bwd = h.dl + rowsp * HEAD_TILE * 2 * h.parts + dzp;
    return std::max(h.picked + ((rowsp * 4 + 255) & ~(size_t)255), bwd);
}

int launch_head_loss(const Dims &p, const HeadPlan &h, const HeadIn &in, float *ce, float *lse, float *kl, float *tlse,
                     float *logp, void *ws, cudaStream_t s) {
    const __nv_bfloat16 *zp, *wp;
    int st = prepare(p, h, in, ws, &zp, &wp, s);
    if (st != VMOE_OK) return st;
    HeadGemm g = {};
    g.stats = h.stats;
    g.rows = at<int>(ws, h.rows);
    g.vn = h.V;
    g.label = in.label ? at<int>(ws, h.label) : nullptr;
    g.part = at<float2>(ws, h.part);
    g.part2 = at<float2>(ws, h.part2);
    g.picked = at<float>(ws, h.picked);
    if ((st = launch_head_gemm(HEAD_STATS, h, g, zp, wp, nullptr, nullptr, s)) != VMOE_OK) return st;
    Finish f = {};
    f.z = sizes_of(h);
    f.halves = (h.V + 127) / 128;
    f.pitch = (h.V + HEAD_TILE - 1) / HEAD_TILE * 2;
    f.stats = h.stats;
    f.inv_tau = 1.0f / h.tau;
    f.c1 = h.c1;
    f.rows = g.rows;
    f.pos = at<int>(ws, h.pos);
    f.map = at<int>(ws, h.map);
    f.label = at<int>(ws, h.label);
    f.part = g.part;
    f.part2 = g.part2;
    f.picked = g.picked;
    f.tidx = in.tidx;
    f.tlogit = in.tlogit;
    f.ce = ce;
    f.lse = lse;
    f.kl = kl;
    f.tlse = tlse;
    f.logp = logp;
    trace_before(s, "head_finish");
    const dim3 grid((h.N + HF_ROWS - 1) / HF_ROWS, h.T);
    st = p.bf16 ? launch_kernel(head_finish_kernel<__nv_bfloat16>, grid, dim3(HG_THREADS), 0, s, f, (const __nv_bfloat16 *)in.z,
                                (const __nv_bfloat16 *)in.w)
                : launch_kernel(head_finish_kernel<float>, grid, dim3(HG_THREADS), 0, s, f, (const float *)in.z, (const float *)in.w);
    trace_after(s);
    return st;
}

int launch_head_loss_bwd(const Dims &p, const HeadPlan &h, const HeadIn &in, const float *ce, const float *lse,
                         const float *tlse, const float *logp, const float *dce, const float *dlse, const float *dkl, void *dz,
                         void *dw, void *ws, cudaStream_t s) {
    const __nv_bfloat16 *zp, *wp;
    int st = prepare(p, h, in, ws, &zp, &wp, s);
    if (st != VMOE_OK) return st;
    const Sizes z = sizes_of(h);
    const int *rows = at<int>(ws, h.rows), *map = at<int>(ws, h.map);
    Coef c = {};
    c.z = z;
    c.inv_tau = 1.0f / h.tau;
    c.one = h.stats == 1;
    c.rows = rows;
    c.map = map;
    c.label = in.label;
    c.tidx = in.tidx;
    c.tlogit = in.tlogit;
    c.ce = ce;
    c.lse = lse;
    c.tlse = tlse;
    c.dce = dce;
    c.dlse = dlse;
    c.dkl = dkl;
    c.coef = at<float4>(ws, h.coef);
    c.at_label = at<float>(ws, h.at_label);
    trace_before(s, "head_coef");
    st = launch_kernel(head_coef_kernel, dim3((h.N + HG_THREADS - 1) / HG_THREADS, h.T), dim3(HG_THREADS), 0, s, c);
    trace_after(s);
    if (st != VMOE_OK) return st;
    __nv_bfloat16 *dl = at<__nv_bfloat16>(ws, h.dl);
    HeadGemm g = {};
    g.stats = h.stats;
    g.rows = rows;
    g.label = in.label ? at<int>(ws, h.label) : nullptr;
    g.coef = c.coef;
    g.at_label = c.at_label;
    g.splits = h.splits;
    for (int v0 = 0; v0 < h.V; v0 += h.piece) {
        g.v0 = v0;
        g.vn = std::min(h.piece, h.V - v0);
        g.first = v0 == 0;
        g.out = nullptr;
        if ((st = launch_head_gemm(HEAD_DLOGITS, h, g, zp, wp, dl, nullptr, s)) != VMOE_OK) return st;
        if (in.tidx && dkl) {
            Patch f = {};
            f.z = z;
            f.v0 = v0;
            f.vn = g.vn;
            f.piece = h.piece;
            f.parts = h.parts;
            f.tau = h.tau;
            f.inv_tau = c.inv_tau;
            f.rows = rows;
            f.map = map;
            f.label = in.label;
            f.tidx = in.tidx;
            f.tlogit = in.tlogit;
            f.ce = ce;
            f.lse = lse;
            f.tlse = tlse;
            f.logp = logp;
            f.dce = dce;
            f.dlse = dlse;
            f.dkl = dkl;
            f.dl = dl;
            trace_before(s, "head_patch");
            st = launch_kernel(head_patch_kernel, dim3((h.N + 7) / 8, h.T), dim3(HG_THREADS), 0, s, f);
            trace_after(s);
            if (st != VMOE_OK) return st;
        }
        if (dz) {
            g.out = at<float>(ws, h.dzp);
            if ((st = launch_head_gemm(HEAD_DZ, h, g, zp, wp, dl, nullptr, s)) != VMOE_OK) return st;
        }
        if (dw) {
            g.out = (float *)dw;
            if ((st = launch_head_gemm(HEAD_DW, h, g, zp, wp, dl, (__nv_bfloat16 *)dw, s)) != VMOE_OK) return st;
        }
    }
    if (!dz) return VMOE_OK;
    trace_before(s, "head_dz_join");
    const long long blocks = ((long long)h.T * h.N * (h.d / 8) + HG_THREADS - 1) / HG_THREADS;
    const dim3 grid((unsigned)std::min(blocks, 16LL * num_sms()));
    const int *pos = at<int>(ws, h.pos);
    const float *parts = at<float>(ws, h.dzp);
    st = p.bf16 ? launch_kernel(head_dz_kernel<__nv_bfloat16>, grid, dim3(HG_THREADS), 0, s, z, h.splits, pos, parts, (__nv_bfloat16 *)dz)
                : launch_kernel(head_dz_kernel<float>, grid, dim3(HG_THREADS), 0, s, z, h.splits, pos, parts, (float *)dz);
    trace_after(s);
    return st;
}

}  // namespace vmoe

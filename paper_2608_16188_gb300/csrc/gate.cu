// gate.cu -- the choice of experts from router logits (Section 2.1: tokens go to their most relevant
// experts; Challenge #1 in Section 1: capacity limits) with scores, a bias that balances the choice and not the
// gates, and groups of experts, and the gradient through its gates.
//
//   s_e = sigmoid(l_e), or the softmax of the row;  c_e = s_e + b_e
//   a group's score: the sum of its `top` largest c; the `kept` groups of the largest scores are open
//   choices: the k largest c in open groups;  gate_j = scale s_j / sum_i s_i  (scale s_j without renormalisation)
//
// The choices are whole numbers that everything behind them follows, and two experts' c may be closer than the
// rounding of fp32.  They are defined by exact arithmetic, equal ones to the lower index: c is computed in fp32 with
// a bound on its error, and where a choice's runner-up is within it, those experts alone are compared in 64 bits (a
// row in a thousand at 256 experts).  Without a bias the order is that of the logits, which needs neither.
//
// gate_rows: a warp a row, lane l holding experts l, l + 32, ...; a CTA's tile of rows also counts its choices by
// (choice, expert).  gate_slots: the tile's first place for every (choice, expert) is the sum of the counts of all
// tiles' earlier choices and of the earlier tiles' same choice; a warp then ranks a choice of the tile 32 rows at a
// time.  Slots are those of vmoe_route: choice by choice, in token order.  No floating-point sum depends on an order of
// arrival, and the integer atomics' order does not show.
#include <math.h>

#include "gate.cuh"

namespace vmoe {
namespace {

constexpr int GT_THREADS = 256, GT_WARPS = GT_THREADS / 32;
constexpr unsigned FULL = 0xffffffffu;

// The largest c is within this of another: the two may be in either order.  s: expf and the division are off by
// 2^-21 of it in all, the sum of a softmax's row by as much; c: its rounding.
__device__ __forceinline__ float near_of(float s, float c) { return 2e-6f * s + 1.3e-7f * fabsf(c); }

// c in 64 bits; softmax: top the row's largest logit, inv 1 / its sum
__device__ __noinline__ double exact_value(float x, float b, int softmax, double top, double inv) {
    const double s = softmax ? exp((double)x - top) * inv : 1.0 / (1.0 + exp(-(double)x));
    return s + (double)b;
}

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

// M experts a lane: E <= 32 M.
template <int M>
__global__ void __launch_bounds__(GT_THREADS)
gate_rows_kernel(Dims p, Gating g, int rows, const float *__restrict__ logits, const float *__restrict__ sbias,
                 const uint8_t *__restrict__ mask, int32_t *__restrict__ out_idx, float *__restrict__ out_gate,
                 int32_t *__restrict__ hist) {
    extern __shared__ __align__(16) uint8_t gt_smem[];
    const int E = p.E, k = p.k, N = p.N, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double *cd = reinterpret_cast<double *>(gt_smem) + warp * 32 * M;                // [32 M] a warp: c in 64 bits
    float *cf = reinterpret_cast<float *>(gt_smem + GT_WARPS * 32 * M * 8) + warp * 64 * M;  // [32 M] c, [32 M] the groups' scores
    float *gs = cf + 32 * M;
    int *count = reinterpret_cast<int *>(gt_smem + GT_WARPS * 32 * M * 16);          // [k][E]
    const int t = blockIdx.y, n0 = blockIdx.x * rows, n1 = min(N, n0 + rows), gsize = E / g.groups;
    const bool softmax = g.score == VMOE_SCORE_SOFTMAX, grouped = g.groups > 1;
    const bool by_logit = sbias == nullptr;                      // the order of c is that of the logits
    const bool group_by_logit = by_logit && g.top == 1;
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) count[i] = 0;
    pdl_wait();
    float b[M];
#pragma unroll
    for (int i = 0; i < M; ++i) b[i] = sbias && lane + 32 * i < E ? sbias[(long long)t * E + lane + 32 * i] : 0.0f;
    __syncthreads();
    for (int n = n0 + warp; n < n1; n += GT_WARPS) {
        const long long tn = (long long)t * N + n;
        const bool takes = mask == nullptr || mask[tn] != 0;
        float x[M], s[M], c[M], mx = -INFINITY;
        bool on[M];
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const int e = lane + 32 * i;
            x[i] = takes && e < E ? __ldg(logits + tn * E + e) : -INFINITY;
            if (!(fabsf(x[i]) < INFINITY)) x[i] = -INFINITY;
            on[i] = x[i] > -INFINITY && fabsf(b[i]) < INFINITY;  // what is not finite is off
            mx = fmaxf(mx, x[i]);
        }
        mx = softmax ? warp_max(mx) : 0.0f;
        float sum = 1.0f;
        if (softmax) {
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < M; ++i) {
                s[i] = x[i] > -INFINITY ? expf(x[i] - mx) : 0.0f;
                sum += s[i];
            }
            sum = warp_sum(sum);
        }
#pragma unroll
        for (int i = 0; i < M; ++i) {
            s[i] = softmax ? s[i] / sum : 1.0f / (1.0f + expf(-x[i]));
            c[i] = on[i] ? (by_logit ? x[i] : s[i] + b[i]) : -INFINITY;
        }
        double top64 = mx, inv64 = 0.0;
        auto row64 = [&]() {  // the row's sum in 64 bits, once it is needed
            if (!softmax || inv64 != 0.0) return;
            double v = 0.0;
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (x[i] > -INFINITY) v += exp((double)x[i] - top64);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
            inv64 = 1.0 / v;
        };
        if (grouped) {
            // a lane a group: the sum of its `top` largest values, its rank among the groups
            float err = 0.0f;
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const int e = lane + 32 * i;
                if (e >= E) continue;
                const float v = !on[i] ? -INFINITY : group_by_logit ? x[i] : s[i] + b[i];
                cf[e] = v;
                if (on[i] && !group_by_logit) err = fmaxf(err, near_of(s[i], v));
            }
            err = 2.0f * g.top * warp_max(err);
            __syncwarp();
            for (int q = lane; q < g.groups; q += 32) {
                float a = -INFINITY, a2 = -INFINITY;
                for (int i = 0; i < gsize; ++i) {
                    const float v = cf[q * gsize + i];
                    a2 = fmaxf(a2, fminf(a, v));
                    a = fmaxf(a, v);
                }
                gs[q] = g.top == 2 ? a + a2 : a;
            }
            __syncwarp();
            // the groups before q in the order: a larger score, or the same and a lower index
            auto rank_of = [&](int q, auto *score) {
                int r = 0;
                for (int o = 0; o < g.groups; ++o) r += score[o] > score[q] || (score[o] == score[q] && o < q);
                return r;
            };
            float in = INFINITY, out = -INFINITY;
            unsigned open = 0;  // bit q / 32: group q of this lane
            for (int q = lane; q < g.groups; q += 32) {
                const bool kept = rank_of(q, gs) < g.kept;
                open |= (unsigned)kept << (q >> 5);
                if (kept) in = fminf(in, gs[q]);
                else out = fmaxf(out, gs[q]);
            }
            in = -warp_max(-in);
            out = warp_max(out);
            if (!group_by_logit && out > -INFINITY && !(in - out > err)) {
                // all of the same logit and bias: the fp32 values are equal where the exact ones are
                float lo = INFINITY, hi = -INFINITY, blo = INFINITY, bhi = -INFINITY;
#pragma unroll
                for (int i = 0; i < M; ++i)
                    if (on[i]) {
                        lo = fminf(lo, x[i]);
                        hi = fmaxf(hi, x[i]);
                        blo = fminf(blo, b[i]);
                        bhi = fmaxf(bhi, b[i]);
                    }
                if (warp_max(-lo) != -warp_max(hi) || warp_max(-blo) != -warp_max(bhi)) {
                    row64();
#pragma unroll
                    for (int i = 0; i < M; ++i)
                        if (lane + 32 * i < E)
                            cd[lane + 32 * i] = on[i] ? exact_value(x[i], b[i], softmax, top64, inv64) : -INFINITY;
                    __syncwarp();
                    double mine[M];
                    int m = 0;
#pragma unroll
                    for (int i = 0; i < M; ++i) {
                        mine[i] = -INFINITY;
                        const int q = lane + 32 * i;
                        if (q >= g.groups) continue;
                        double a = -INFINITY, a2 = -INFINITY;
                        for (int o = 0; o < gsize; ++o) {
                            const double v = cd[q * gsize + o];
                            a2 = fmax(a2, fmin(a, v));
                            a = fmax(a, v);
                        }
                        mine[i] = g.top == 2 ? a + a2 : a;
                        m = i + 1;
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < M; ++i)
                        if (i < m) cd[lane + 32 * i] = mine[i];
                    __syncwarp();
                    open = 0;
                    for (int q = lane; q < g.groups; q += 32) open |= (unsigned)(rank_of(q, cd) < g.kept) << (q >> 5);
                    __syncwarp();
                }
            }
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const int q = min(lane + 32 * i, E - 1) / gsize;
                const unsigned word = __shfl_sync(FULL, open, q & 31);
                if (!((word >> (q >> 5)) & 1u)) c[i] = -INFINITY;
            }
            __syncwarp();
        }
        // the k largest c in turn
        float my_x = -INFINITY;
        int my_e = -1;
        for (int j = 0; j < k; ++j) {
            float m = c[0];
            int at = 0;
#pragma unroll
            for (int i = 1; i < M; ++i)
                if (c[i] > m) {
                    m = c[i];
                    at = i;
                }
            const float best = warp_max(m);
            if (!(best > -INFINITY)) break;
            float low = best;  // by_logit: equal ones alone
            if (!by_logit) {
                float sb = 0.0f;
#pragma unroll
                for (int i = 0; i < M; ++i)
                    if (i == at && m == best) sb = s[i];
                low -= near_of(warp_max(sb), best);
            }
            auto may_be = [&](int i) { return c[i] > -INFINITY && (by_logit ? c[i] == low : c[i] + near_of(s[i], c[i]) >= low); };
            // whoever may be the largest: one, as a rule
            int mine = 0, e = E;
#pragma unroll
            for (int i = M - 1; i >= 0; --i)
                if (may_be(i)) {
                    ++mine;
                    e = lane + 32 * i;
                }
            if (!by_logit && __reduce_add_sync(FULL, mine) > 1) {
                // the first of them, and whether all have its logit and bias
                const int first = __reduce_min_sync(FULL, e);
                float fx = 0.0f, fb = 0.0f;
#pragma unroll
                for (int i = 0; i < M; ++i)
                    if (lane + 32 * i == first) {
                        fx = x[i];
                        fb = b[i];
                    }
                fx = __shfl_sync(FULL, fx, first & 31);
                fb = __shfl_sync(FULL, fb, first & 31);
                bool same = true;
#pragma unroll
                for (int i = 0; i < M; ++i)
                    if (may_be(i)) same &= x[i] == fx && b[i] == fb;
                if (!__all_sync(FULL, same)) {
                    row64();
                    double v = -INFINITY;
                    e = E;
#pragma unroll
                    for (int i = 0; i < M; ++i)
                        if (may_be(i)) {
                            const double w = exact_value(x[i], b[i], softmax, top64, inv64);
                            if (w > v || e == E) {
                                v = w;
                                e = lane + 32 * i;
                            }
                        }
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) {
                        const double ov = __shfl_xor_sync(FULL, v, o);
                        const int oe = __shfl_xor_sync(FULL, e, o);
                        if (oe < E && (e == E || ov > v || (ov == v && oe < e))) {
                            v = ov;
                            e = oe;
                        }
                    }
                }
            }
            const int chosen = __reduce_min_sync(FULL, e);
            float cx = 0.0f;
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (lane + 32 * i == chosen) {
                    cx = x[i];
                    c[i] = -INFINITY;
                }
            cx = __shfl_sync(FULL, cx, chosen & 31);
            if (lane == j) {
                my_x = cx;
                my_e = chosen;
            }
        }
        // the gates: lanes 0 to k - 1
        const float xmax = warp_max(my_x);
        float w = 0.0f;
        if (my_e >= 0) {
            // exp(x - xmax) is a softmax's ratio, and a sigmoid's where all are so far out that it is exp(x)
            if (softmax && g.renorm) w = expf(my_x - xmax);
            else if (softmax) w = expf(my_x - mx) / sum;
            else if (g.renorm && xmax < -60.0f) w = expf(my_x - xmax);
            else w = 1.0f / (1.0f + expf(-my_x));
        }
        const float mass = warp_sum(w);
        if (lane < k) {
            out_idx[tn * k + lane] = my_e;
            out_gate[tn * k + lane] = my_e < 0 ? 0.0f : g.renorm ? g.scale * (w / mass) : g.scale * w;
            if (my_e >= 0) atomicAdd(count + lane * E + my_e, 1);
        }
    }
    __syncthreads();
    int32_t *h = hist + ((long long)t * gridDim.x + blockIdx.x) * k * E;
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) h[i] = count[i];
}

__global__ void __launch_bounds__(GT_THREADS)
gate_slots_kernel(Dims p, int rows, const int32_t *__restrict__ idx, const int32_t *__restrict__ hist,
                  int32_t *__restrict__ slot, int32_t *__restrict__ load, int32_t *__restrict__ demand) {
    extern __shared__ int gt_base[];  // [k][E]: the next place of each (choice, expert); then [k][E] whole counts
    const int E = p.E, k = p.k, N = p.N, t = blockIdx.y, tiles = gridDim.x, tile = blockIdx.x;
    int *all = gt_base + k * E;
    pdl_wait();
    const int32_t *h = hist + (long long)t * tiles * k * E;
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) {
        int before = 0, total = 0;
#pragma unroll 8
        for (int q = 0; q < tiles; ++q) {
            const int v = h[(long long)q * k * E + i];
            if (q < tile) before += v;
            total += v;
        }
        gt_base[i] = before;
        all[i] = total;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += GT_THREADS) {
        int run = 0;
        for (int j = 0; j < k; ++j) {
            gt_base[j * E + e] += run;
            run += all[j * E + e];
        }
        if (tile == 0) {
            load[(long long)t * E + e] = min(run, p.C);
            if (demand) demand[(long long)t * E + e] = run;
        }
    }
    __syncthreads();
    const int j = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (j >= k) return;
    int *next = gt_base + j * E;
    const int n0 = tile * rows, n1 = min(N, n0 + rows);
    for (int n = n0; n < n1; n += 32) {
        const long long at = ((long long)t * N + n + lane) * k + j;
        const int e = n + lane < n1 ? idx[at] : -1;
        const unsigned peers = __match_any_sync(FULL, e);
        const int before = __popc(peers & ((1u << lane) - 1u));
        const int base = e >= 0 ? next[e] : 0;
        __syncwarp();
        if (e >= 0 && before == 0) next[e] = base + __popc(peers);
        __syncwarp();
        if (n + lane < n1) slot[at] = e >= 0 && base + before < p.C ? base + before : -1;
    }
}

// b_e += rate sign(mean - count_e): E count_e against the sum, both whole.
__global__ void gate_bias_kernel(int E, const int32_t *__restrict__ demand, float rate, float *__restrict__ bias) {
    pdl_wait();
    const int t = blockIdx.x, lane = threadIdx.x;
    const int32_t *c = demand + (long long)t * E;
    long long sum = 0;
    for (int e = lane; e < E; e += 32) sum += c[e];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
    for (int e = lane; e < E; e += 32) {
        const long long mine = (long long)c[e] * E;
        if (mine != sum) bias[(long long)t * E + e] += mine < sum ? rate : -rate;
    }
}

// ---------------------------------------------------------------------------
// The gradient through the gates, choices held fixed: with r_j = gate_j / scale and m = sum_i r_i dgate_i
//   sigmoid:  dl_j = gate_j (1 - s_j) (dgate_j - m),  without renormalisation gate_j (1 - s_j) dgate_j
//   softmax:  dl_j = gate_j (dgate_j - m),  without renormalisation dl_e = scale p_e (dgate_e - m), all e
// A warp a token: dgate_j = <dY, Ye[e_j, s_j]> streams dY and the chosen rows.
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

template <typename T, int KMAX>
__global__ void __launch_bounds__(GT_THREADS)
gate_grad_kernel(Dims p, Gating g, const float *__restrict__ logits, const int32_t *__restrict__ idx,
                 const float *__restrict__ gate, const int32_t *__restrict__ slot, const T *__restrict__ dy,
                 const T *__restrict__ ye, float *__restrict__ dgate, float *__restrict__ dlogits) {
    const int lane = threadIdx.x & 31, d = p.d, E = p.E, k = p.k;
    const long long tn = (long long)blockIdx.x * GT_WARPS + (threadIdx.x >> 5);
    pdl_wait();
    if (tn >= (long long)p.T * p.N) return;
    const int t = (int)(tn / p.N);
    int ei[KMAX], sl[KMAX];
    float gt[KMAX], dg[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        ei[j] = j < k ? idx[tn * k + j] : -1;
        sl[j] = j < k ? slot[tn * k + j] : -1;
        gt[j] = j < k ? gate[tn * k + j] : 0.0f;
        dg[j] = 0.0f;
    }
    for (int v = lane * 8; v < d; v += 256) {
        float fa[8];
        load8<T>(dy + tn * d + v, fa);
#pragma unroll
        for (int j = 0; j < KMAX; ++j) {
            if (sl[j] < 0) continue;
            float fb[8];
            load8<T>(ye + (((long long)t * E + ei[j]) * p.C + sl[j]) * d + v, fb);
#pragma unroll
            for (int q = 0; q < 8; ++q) dg[j] = fmaf(fa[q], fb[q], dg[j]);
        }
    }
    float m = 0.0f, mine = 0.0f;
    bool some = false;
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        dg[j] = warp_sum(dg[j]);
        if (lane == j) mine = dg[j];
        if (ei[j] < 0) continue;
        some = true;
        m = fmaf(gt[j] / g.scale, dg[j], m);
    }
    if (lane < k) dgate[tn * k + lane] = mine;
    const bool add = (p.flags & VMOE_DLOGITS_ADD) != 0;
    const float *l = logits + tn * E;
    float *dl = dlogits + tn * E;
    if (g.score == VMOE_SCORE_SOFTMAX && !g.renorm && some) {
        float mx = -INFINITY, sum = 0.0f;
        for (int e = lane; e < E; e += 32)
            if (fabsf(l[e]) < INFINITY) mx = fmaxf(mx, l[e]);
        mx = warp_max(mx);
        for (int e = lane; e < E; e += 32)
            if (fabsf(l[e]) < INFINITY) sum += expf(l[e] - mx);
        sum = warp_sum(sum);
        for (int e = lane; e < E; e += 32) {
            float ge = 0.0f;
#pragma unroll
            for (int j = 0; j < KMAX; ++j)
                if (ei[j] == e) ge = dg[j];
            float v = fabsf(l[e]) < INFINITY ? g.scale * (expf(l[e] - mx) / sum) * (ge - m) : 0.0f;
            if (add) v += dl[e];
            dl[e] = v;
        }
        return;
    }
    float c[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
        c[j] = 0.0f;
        if (ei[j] < 0) continue;
        c[j] = gt[j] * (g.renorm ? dg[j] - m : dg[j]);
        if (g.score == VMOE_SCORE_SIGMOID) c[j] *= 1.0f / (1.0f + expf(l[ei[j]]));
    }
    for (int e = lane; e < E; e += 32) {
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < KMAX; ++j)
            if (ei[j] == e) v = c[j];
        if (add) v += dl[e];
        dl[e] = v;
    }
}

template <typename T, int KMAX>
int launch_grad(const Dims &p, const Gating &g, const float *logits, const int32_t *idx, const float *gate,
                const int32_t *slot, const void *dy, const void *ye, float *dgate, float *dlogits, cudaStream_t s) {
    const long long blocks = ((long long)p.T * p.N + GT_WARPS - 1) / GT_WARPS;
    return launch_kernel(gate_grad_kernel<T, KMAX>, dim3((unsigned)blocks), dim3(GT_THREADS), 0, s, p, g, logits, idx, gate,
                         slot, (const T *)dy, (const T *)ye, dgate, dlogits);
}
template <typename T>
int launch_grad_k(const Dims &p, const Gating &g, const float *logits, const int32_t *idx, const float *gate,
                  const int32_t *slot, const void *dy, const void *ye, float *dgate, float *dlogits, cudaStream_t s) {
    if (p.k <= 1) return launch_grad<T, 1>(p, g, logits, idx, gate, slot, dy, ye, dgate, dlogits, s);
    if (p.k <= 2) return launch_grad<T, 2>(p, g, logits, idx, gate, slot, dy, ye, dgate, dlogits, s);
    if (p.k <= 4) return launch_grad<T, 4>(p, g, logits, idx, gate, slot, dy, ye, dgate, dlogits, s);
    return launch_grad<T, 8>(p, g, logits, idx, gate, slot, dy, ye, dgate, dlogits, s);
}

// Rows of a tile: 64, more where a task would have over 128 tiles.
int tile_rows(int N) {
    int rows = 64;
    while ((N + rows - 1) / rows > 128) rows *= 2;
    return rows;
}

template <int M>
int launch_rows(const Dims &p, const Gating &g, int rows, const float *logits, const float *sbias, const uint8_t *mask,
                int32_t *idx, float *gate, int32_t *hist, cudaStream_t s) {
    const size_t smem = (size_t)GT_WARPS * 32 * M * 16 + (size_t)p.k * p.E * 4;  // at most 40 KB
    return launch_kernel(gate_rows_kernel<M>, dim3((p.N + rows - 1) / rows, p.T), dim3(GT_THREADS), smem, s, p, g, rows,
                         logits, sbias, mask, idx, gate, hist);
}

}  // namespace

size_t gate_workspace(const Dims &p) {
    const int rows = tile_rows(p.N);
    return (size_t)p.T * ((p.N + rows - 1) / rows) * p.k * p.E * 4;
}

int launch_gate(const Dims &p, const Gating &g, const float *logits, const float *sbias, const uint8_t *mask, int32_t *idx,
                float *gate, int32_t *slot, int32_t *load, int32_t *demand, int32_t *hist, cudaStream_t s) {
    const int rows = tile_rows(p.N);
    trace_before(s, "gate_rows");
    int st = p.E <= 32    ? launch_rows<1>(p, g, rows, logits, sbias, mask, idx, gate, hist, s)
             : p.E <= 64  ? launch_rows<2>(p, g, rows, logits, sbias, mask, idx, gate, hist, s)
             : p.E <= 128 ? launch_rows<4>(p, g, rows, logits, sbias, mask, idx, gate, hist, s)
                          : launch_rows<8>(p, g, rows, logits, sbias, mask, idx, gate, hist, s);
    trace_after(s);
    if (st != VMOE_OK) return st;
    trace_before(s, "gate_slots");
    st = launch_kernel(gate_slots_kernel, dim3((p.N + rows - 1) / rows, p.T), dim3(GT_THREADS), (size_t)p.k * p.E * 8, s, p,
                       rows, idx, hist, slot, load, demand);
    trace_after(s);
    return st;
}

int launch_gate_grad(const Dims &p, const Gating &g, const float *logits, const int32_t *idx, const float *gate,
                     const int32_t *slot, const void *dy, const void *ye, float *dgate, float *dlogits, cudaStream_t s) {
    trace_before(s, "gate_grad");
    const int st = p.bf16 ? launch_grad_k<__nv_bfloat16>(p, g, logits, idx, gate, slot, dy, ye, dgate, dlogits, s)
                          : launch_grad_k<float>(p, g, logits, idx, gate, slot, dy, ye, dgate, dlogits, s);
    trace_after(s);
    return st;
}

int launch_gate_bias(const Dims &p, const int32_t *demand, float rate, float *bias, cudaStream_t s) {
    trace_before(s, "gate_bias");
    const int st = launch_kernel(gate_bias_kernel, dim3(p.T), dim3(32), 0, s, p.E, demand, rate, bias);
    trace_after(s);
    return st;
}

}  // namespace vmoe

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
// a bound on its error, and where a choice's runner-up is within it, those experts alone are compared in 64 bits (four
// rows in ten thousand at 256 experts).  Without a bias the order is that of the logits, which needs neither.
//
// gate_fast: a row on a few lanes, in fp32; gate_rows: a warp a row, for groups of odd sizes.  A CTA's tile of rows also
// counts its choices by (choice, expert).  gate_slots: the tile's first place for every (choice, expert) is the sum of
// the counts of all tiles' earlier choices and of the earlier tiles' same choice; a warp then ranks a choice of the tile
// 32 rows at a time.  Slots are those of vmoe_route: choice by choice, in token order.  No floating-point sum depends on an order of
// arrival, and the integer atomics' order does not show.
#include <math.h>

#include <algorithm>

#include "gate.cuh"

namespace vmoe {
namespace {

constexpr int GT_THREADS = 256, GT_WARPS = GT_THREADS / 32;
constexpr unsigned FULL = 0xffffffffu;

// The largest c is within this of another: the two may be in either order.  s: expf, the sum and the division are off by
// 1e-6 of it in all, x - max's rounding by 6e-8 |x - max|, at most 87 of them before s is 0; c: its rounding.
__device__ __forceinline__ float near_of(float s, float c) { return 8e-6f * s + 1.3e-7f * fabsf(c); }

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

// A row's choices: lane j has the j-th expert and its logit, -1 and -inf where there is none.  mx, sum: the softmax's
// largest logit and sum of exponentials.
struct Choice {
    int e;
    float x, mx, sum;
};

// One row by a whole warp, whatever the groups' size, M experts a lane (E <= 32 M), with the comparisons in 64 bits where
// fp32 leaves them open.  cd [32 M], cf [32 M], gs [32 M]: this warp's scratch.
template <int M>
__device__ __noinline__ Choice choose_row(const Dims &p, const Gating &g, int t, long long tn, const float *__restrict__ logits,
                                          const float *__restrict__ sbias, double *cd, float *cf, float *gs) {
    const int E = p.E, k = p.k, lane = threadIdx.x & 31, gsize = E / g.groups;
    const bool softmax = g.score == VMOE_SCORE_SOFTMAX, grouped = g.groups > 1;
    const bool by_logit = sbias == nullptr;  // the order of c is that of the logits
    const bool group_by_logit = by_logit && g.top == 1;
    float x[M], s[M], c[M], b[M], mx = -INFINITY;
    bool on[M];
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int e = lane + 32 * i;
        x[i] = e < E ? __ldg(logits + tn * E + e) : -INFINITY;
        b[i] = sbias && e < E ? __ldg(sbias + (long long)t * E + e) : 0.0f;
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
    Choice r;
    r.x = -INFINITY;
    r.e = -1;
    r.mx = mx;
    r.sum = sum;
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
            r.x = cx;
            r.e = chosen;
        }
    }
    return r;
}

// Gate of lane j's choice; `size` lanes of the warp hold a row's.
__device__ __forceinline__ float gate_of(const Gating &g, const Choice &r, int size) {
    float xmax = r.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < size) xmax = fmaxf(xmax, __shfl_xor_sync(FULL, xmax, o));
    const bool softmax = g.score == VMOE_SCORE_SOFTMAX;
    float w = 0.0f;
    if (r.e >= 0) {
        // exp(x - xmax) is a softmax's ratio, and a sigmoid's where all are so far out that it is exp(x)
        if (softmax && !g.renorm) w = expf(r.x - r.mx) / r.sum;
        else if (softmax || (g.renorm && xmax < -60.0f)) w = expf(r.x - xmax);
        else w = 1.0f / (1.0f + expf(-r.x));
    }
    float mass = w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < size) mass += __shfl_xor_sync(FULL, mass, o);
    return r.e < 0 ? 0.0f : g.renorm ? g.scale * (w / mass) : g.scale * w;
}

constexpr size_t row_scratch(int M) { return (size_t)GT_WARPS * 32 * M * 16; }

// Groups of a number of experts that is no power of two or below a lane's in gate_fast.
template <int M>
__global__ void __launch_bounds__(GT_THREADS, 3)
gate_rows_kernel(Dims p, Gating g, int rows, const float *__restrict__ logits, const float *__restrict__ sbias,
                 const uint8_t *__restrict__ mask, int32_t *__restrict__ out_idx, float *__restrict__ out_gate,
                 int32_t *__restrict__ hist) {
    extern __shared__ __align__(16) uint8_t gt_smem[];
    const int E = p.E, k = p.k, N = p.N, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double *cd = reinterpret_cast<double *>(gt_smem) + warp * 64 * M;
    float *cf = reinterpret_cast<float *>(cd + 32 * M), *gs = cf + 32 * M;
    int *count = reinterpret_cast<int *>(gt_smem + row_scratch(M));  // [k][E]
    const int t = blockIdx.y, n0 = blockIdx.x * rows, n1 = min(N, n0 + rows);
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) count[i] = 0;
    pdl_wait();
    pdl_launch_dependents();
    __syncthreads();
    for (int n = n0 + warp; n < n1; n += GT_WARPS) {
        const long long tn = (long long)t * N + n;
        Choice r = {-1, -INFINITY, 0.0f, 1.0f};
        if (mask == nullptr || mask[tn] != 0) r = choose_row<M>(p, g, t, tn, logits, sbias, cd, cf, gs);
        const float gate = gate_of(g, r, 32);
        if (lane < k) {
            out_idx[tn * k + lane] = r.e;
            out_gate[tn * k + lane] = gate;
            if (r.e >= 0) atomicAdd(count + lane * E + r.e, 1);
        }
    }
    __syncthreads();
    int32_t *h = hist + ((long long)t * gridDim.x + blockIdx.x) * k * E;
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) h[i] = count[i];
}

__device__ __forceinline__ float ex2(float v) {
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
}
__device__ __forceinline__ float rcp(float v) {
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
}
__device__ __forceinline__ float redux_max(float v) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// The largest of this lane's half of the warp, for two rows a warp: 8 x 60000 of 64 experts, k 8, 8 groups, 350 -> 316 us
// against four exchanges with their comparisons.
__device__ __forceinline__ float redux_max_half(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "r"((threadIdx.x & 16) ? 0xffff0000u : 0x0000ffffu));
    return r;
}

// V values of a lane, the largest first; at: where each came from, 4 bits apiece (a network of compare-exchanges).
template <int V>
__device__ __forceinline__ unsigned sort_lane(float (&h)[V]) {
    int at[V];
#pragma unroll
    for (int i = 0; i < V; ++i) at[i] = i;
    auto order = [&](int i, int j) {
        const bool swap = h[j] > h[i];
        const float hi = swap ? h[j] : h[i], lo = swap ? h[i] : h[j];
        const int ai = swap ? at[j] : at[i], aj = swap ? at[i] : at[j];
        h[i] = hi, h[j] = lo, at[i] = ai, at[j] = aj;
    };
    auto merge4 = [&](int i) {
        order(i, i + 1), order(i + 2, i + 3), order(i, i + 2), order(i + 1, i + 3), order(i + 1, i + 2);
    };
    merge4(0);
    if constexpr (V == 8) {
        merge4(4);
        order(0, 4), order(1, 5), order(2, 6), order(3, 7);
        order(2, 4), order(3, 5);
        order(1, 2), order(3, 4), order(5, 6);
    }
    unsigned r = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) r |= (unsigned)at[i] << (4 * i);
    return r;
}

// A row on L lanes, V experts in a row each (L V >= E), 32 / L rows a warp, the next ones' logits in flight; no group, or
// groups of a power of two of experts, at least V of them.  A lane sorts its values once; a choice is then the largest of
// the lanes' first values, and its lane moves up.  c is formed with the approximate exponential and reciprocal; a row
// with two of the first k + 1 values, or an open and a shut group, closer than their error (or equal) is done again by
// choose_row behind the loop:
//   sigmoid: the exponential is off by 2^-22 + |x| 2^-23.5 relative, which e / (1 + e)^2 <= 1 / 4 and |x| e / (1 + e)^2 <=
//   0.23 take to 8e-8 of 1 in s, the reciprocal and the sum add 1.8e-7 s; softmax: exponential, sum and reciprocal 1e-6 s
//   and 6e-8 |x - max| s, at most 87 of them before s is 0: 8e-6 s; c's rounding 6e-8 |c|.
template <int L, int V>
__global__ void __launch_bounds__(GT_THREADS, 4)
gate_fast_kernel(Dims p, Gating g, int rows, const float *__restrict__ logits, const float *__restrict__ sbias,
                 const uint8_t *__restrict__ mask, int32_t *__restrict__ out_idx, float *__restrict__ out_gate,
                 int32_t *__restrict__ hist) {
    constexpr int RW = 32 / L, M = L * V / 32 > 0 ? L * V / 32 : 1;
    constexpr float LOG2E = 1.4426950408889634f;
    extern __shared__ __align__(16) uint8_t gt_smem[];
    const int E = p.E, k = p.k, N = p.N, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *count = reinterpret_cast<int *>(gt_smem + row_scratch(M));  // [k][E]
    unsigned *again = reinterpret_cast<unsigned *>(count + k * E);   // a bit a row of the tile
    int4 *wait_of = reinterpret_cast<int4 *>(gt_smem + (size_t)warp * 512 * M);  // a warp's scratch, which choose_row has behind the loop
    int2 *mine_of = reinterpret_cast<int2 *>(wait_of + 32);
    const int t = blockIdx.y, n0 = blockIdx.x * rows, n1 = min(N, n0 + rows), gsize = E / g.groups;
    const int sub = lane / L, sl = lane % L, e0 = sl * V, mine = e0 / gsize, glanes = gsize / V;
    const bool softmax = g.score == VMOE_SCORE_SOFTMAX, by_logit = sbias == nullptr, group_by_logit = by_logit && g.top == 1;
    const bool scored = !by_logit || (g.groups > 1 && !group_by_logit);  // s is needed for the choice
    const float *row = logits + (long long)t * N * E;
    for (int i = threadIdx.x; i < k * E + (rows + 31) / 32; i += GT_THREADS) count[i] = 0;
    pdl_wait();
    pdl_launch_dependents();
    float b[V], bmax = 0.0f;  // -inf: off
#pragma unroll
    for (int i = 0; i < V; ++i) {
        b[i] = sbias && e0 + i < E ? __ldg(sbias + (long long)t * E + e0 + i) : 0.0f;
        if (fabsf(b[i]) < INFINITY) bmax = fmaxf(bmax, fabsf(b[i]));
        else b[i] = -INFINITY;
    }
    bmax = warp_max(bmax);
    __syncthreads();
    float next[V];
    bool next_in = false;
    auto load = [&](int n) {
        next_in = n < n1 && (mask == nullptr || mask[(long long)t * N + n] != 0);
        const float *src = row + (long long)n * E + e0;
        if (V % 4 == 0 && E % 4 == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (n < n1 && e0 + i < E) v = __ldg(reinterpret_cast<const float4 *>(src + i));
                next[i] = v.x, next[i + 1] = v.y, next[i + 2] = v.z, next[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) next[i] = n < n1 && e0 + i < E ? __ldg(src + i) : -INFINITY;
        }
    };
    // choice j of token n (-1: none; -2: not now): its gate, out and counted
    auto finish = [&](int e, int n, float mx, float sum, int j) {
        Choice r;
        r.e = e;
        r.x = e >= 0 ? __ldg(row + (long long)n * E + e) : -INFINITY;
        r.mx = mx;
        r.sum = sum;
        const float gate = gate_of(g, r, L < 8 ? L : 8);
        if (j < k && e != -2) {
            const long long o = ((long long)t * N + n) * k + j;
            out_idx[o] = e;
            out_gate[o] = gate;
            if (e >= 0) atomicAdd(count + j * E + e, 1);
        }
    };
    int batch = 0;
    load(n0 + warp * RW + sub);
    const float rel = softmax ? 8e-6f : 3e-7f, abs1 = softmax ? 0.0f : 1e-7f;
    for (int base = n0 + warp * RW; base < n1; base += GT_WARPS * RW) {
        const int n = base + sub;
        float c[V], mx = 0.0f, sum = 1.0f, smax = 1.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = next_in && fabsf(next[i]) < INFINITY ? next[i] : -INFINITY;
        load(n + GT_WARPS * RW);
        if (softmax && (scored || !g.renorm)) {
            mx = c[0];
#pragma unroll
            for (int i = 1; i < V; ++i) mx = fmaxf(mx, c[i]);
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, o));
            mx = fmaxf(mx, -3.4028235e38f);  // a row of nothing: exponentials of -inf, not of a NaN
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) sum += g.renorm ? ex2((c[i] - mx) * LOG2E) : expf(c[i] - mx);
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
            smax = rcp(sum);
        }
        const float before = softmax && (scored || !g.renorm) ? mx : 0.0f;
        if (scored) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = softmax ? ex2((c[i] - before) * LOG2E) * smax : rcp(1.0f + ex2(-c[i] * LOG2E));
                c[i] = c[i] > -INFINITY ? s + b[i] : -INFINITY;
            }
        }
        // the error of a value, from s <= smax, c + bmax
        auto tol = [&](float v) { return fmaf(rel, fminf(smax, v + bmax), fmaf(1.2e-7f, fabsf(v), abs1)); };
        bool open = false;  // whether two values are too close for fp32
        if (g.groups > 1) {
            float a = c[0], a2 = -INFINITY;
#pragma unroll
            for (int i = 1; i < V; ++i) {
                a2 = fmaxf(a2, fminf(a, c[i]));
                a = fmaxf(a, c[i]);
            }
            for (int o = 1; o < glanes; o <<= 1) {
                const float oa = __shfl_xor_sync(FULL, a, o), oa2 = __shfl_xor_sync(FULL, a2, o);
                a2 = fmaxf(fminf(a, oa), fmaxf(a2, oa2));
                a = fmaxf(a, oa);
            }
            const float score = g.top == 2 ? a + a2 : a;
            // the smallest of the `kept` largest scores, and the largest of the others; equal ones fall together and
            // leave the row open
            auto largest = [&](float v) {
                if constexpr (L == 32) v = redux_max(v);
                else if constexpr (L == 16) v = redux_max_half(v);
                else
                    for (int o = glanes; o < L; o <<= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
                return v;
            };
            float left = mine < g.groups ? score : -INFINITY, in = INFINITY;
            bool tie = false;
            for (int q = 0; q < g.kept; ++q) {
                in = largest(left);
                const unsigned has = __ballot_sync(FULL, left == in) >> (sub * L) & (L == 32 ? FULL : (1u << (L & 31)) - 1u);
                tie |= in > -INFINITY && __popc(has) != glanes;
                if (left == in) left = -INFINITY;
            }
            const float out = largest(left);
            const bool kept = score >= in;
            // fewer whole groups than may be open: the others, with an expert or none, go by their index
            tie |= in == -INFINITY && a > -INFINITY && score == -INFINITY;
            // values at the border are at most |score| + bmax each
            open = tie || (!group_by_logit && out > -INFINITY &&
                           !(in - out > (float)g.top * (tol(fabsf(in) + bmax) + tol(fabsf(out) + bmax))));
            if (by_logit && scored) {  // the choice has the logits' order: the lane's values again, as they came
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float l = n < n1 && e0 + i < E ? __ldg(row + (long long)n * E + e0 + i) : -INFINITY;
                    c[i] = a > -INFINITY && fabsf(l) < INFINITY ? l : -INFINITY;
                }
            }
            if (!kept) {
#pragma unroll
                for (int i = 0; i < V; ++i) c[i] = -INFINITY;
            }
        }
        int my_e = -1;  // lane j: the j-th choice
        bool few = false;
        if (L == 32) {
            // The k-th largest of the lanes' largest values is not above the k-th largest value: what is not below it, a
            // dozen values, goes to shared memory, a value a lane, and each counts how many are above it.
            float m = c[0];
#pragma unroll
            for (int i = 1; i < V; ++i) m = fmaxf(m, c[i]);
            float left = m, least = INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j == k) break;
                least = redux_max(left);
                if (left == least) left = -INFINITY;
            }
            if (!by_logit && least > -INFINITY) least -= 2.0f * tol(least);  // and the next one, if it is near
            least = fmaxf(least, -3.4028235e38f);                            // nothing that is off
            int found = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool take = c[i] >= least;
                const unsigned who = __ballot_sync(FULL, take);
                const int to = found + __popc(who & ((1u << lane) - 1u));
                if (take && to < 32) mine_of[to] = make_int2(__float_as_int(c[i]), e0 + i);
                found += __popc(who);
            }
            few = found <= 32;
            if (few) {
                __syncwarp();
                const int2 own = mine_of[lane];
                const float v = lane < found ? __int_as_float(own.x) : -INFINITY;
                // of k + 1 values in a row none may be near the next (the larger one's error is the smaller's and 3e-6 of the gap)
                const float err = by_logit ? 0.0f : 2.00001f * tol(v);
                int above = 0, near = 0;  // itself among the near ones
                for (int q = 0; q < found; q += 4) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {  // past the last one: -inf
                        const float gap = __shfl_sync(FULL, v, q + u) - v;
                        above += gap > 0.0f;
                        near += fabsf(gap) <= err;
                    }
                }
                open |= lane < found && above <= k && near > 1;
                const unsigned at_rank = lane < found && above < k ? 1u << above : 0u;
                my_e = -1;
                if (at_rank) mine_of[32 + above].y = own.y;
                __syncwarp();
                if (lane < min(k, found)) my_e = mine_of[32 + lane].y;
                __syncwarp();
            }
        }
        if (!few) {
            float value = -INFINITY, last = -INFINITY;  // c of this lane's choice; of the best that was not chosen
            unsigned at = sort_lane<V>(c);
            for (int j = 0; j <= k; ++j) {
                float m = c[0];
                int e = sl;  // the lane that has the largest, the first of equals
                if constexpr (L >= 16) {
                    m = L == 32 ? redux_max(m) : redux_max_half(m);
                    e = __ffs(__ballot_sync(FULL, c[0] == m) >> (L == 32 ? 0 : sub * L)) - 1;
                } else {
#pragma unroll
                    for (int o = L / 2; o > 0; o >>= 1) {
                        const float om = __shfl_xor_sync(FULL, m, o);
                        const int oe = __shfl_xor_sync(FULL, e, o);
                        if (om > m || (om == m && oe < e)) {
                            m = om;
                            e = oe;
                        }
                    }
                }
                if (j == k) {
                    last = m;
                    break;
                }
                const int chosen = e * V + (int)(__shfl_sync(FULL, at, e, L) & 15u);
                if (sl == e) {
#pragma unroll
                    for (int i = 0; i + 1 < V; ++i) c[i] = c[i + 1];
                    c[V - 1] = -INFINITY;
                    at >>= 4;
                }
                if (sl == j && m > -INFINITY) {
                    my_e = chosen;
                    value = m;
                }
            }
            float after = __shfl_down_sync(FULL, value, 1, L);
            if (sl >= k - 1) after = last;
            const float err = by_logit ? 0.0f : tol(value) + tol(after);
            open |= sl < k && after > -INFINITY && !(value - after > err);
        }
        const unsigned redo = __ballot_sync(FULL, open && n < n1) >> (sub * L) & (L == 32 ? FULL : (1u << (L & 31)) - 1u);
        if (redo && sl == 0) atomicOr(again + ((n - n0) >> 5), 1u << ((n - n0) & 31));
        // the gates of four rows of eight lanes at a time
        if (L > 8) {
            if (sl < 8) {
                const int slot = (batch * RW + sub) * 8 + sl;
                wait_of[slot] = make_int4(redo || n >= n1 ? -2 : my_e, n, __float_as_int(mx), __float_as_int(sum));
            }
            if (++batch < L / 8 && base + GT_WARPS * RW < n1) continue;
            __syncwarp();
            const int4 w = lane < batch * RW * 8 ? wait_of[lane] : make_int4(-2, 0, 0, 0);
            batch = 0;
            finish(w.x, w.y, __int_as_float(w.z), __int_as_float(w.w), lane & 7);
            __syncwarp();
        } else {
            finish(redo || n >= n1 ? -2 : my_e, n, mx, sum, sl);
        }
    }
    __syncthreads();
    double *cd = reinterpret_cast<double *>(gt_smem) + warp * 64 * M;
    float *cf = reinterpret_cast<float *>(cd + 32 * M);
    for (int i = warp; i < n1 - n0; i += GT_WARPS) {  // a warp a row
        if (!(again[i >> 5] >> (i & 31) & 1u)) continue;
        const long long tn = (long long)t * N + n0 + i;
        const Choice r = choose_row<M>(p, g, t, tn, logits, sbias, cd, cf, cf + 32 * M);
        const float gate = gate_of(g, r, 32);
        if (lane < k) {
            out_idx[tn * k + lane] = r.e;
            out_gate[tn * k + lane] = gate;
            if (r.e >= 0) atomicAdd(count + lane * E + r.e, 1);
        }
    }
    __syncthreads();
    int32_t *h = hist + ((long long)t * gridDim.x + blockIdx.x) * k * E;
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) h[i] = count[i];
}

// Counts of the tiles before each, in place, and of all of them: hist [T][tiles][k][E], all [T][k][E].  A CTA 32 columns, a
// warp an eighth of the tiles, twice: their sum, then each one's place.
__global__ void __launch_bounds__(GT_THREADS)
gate_scan_kernel(int kE, int tiles, int32_t *__restrict__ hist, int32_t *__restrict__ all) {
    __shared__ int sum[GT_WARPS][32];
    const int t = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    pdl_wait();
    pdl_launch_dependents();
    int32_t *h = hist + (long long)t * tiles * kE + i;
    const int per = (tiles + GT_WARPS - 1) / GT_WARPS, q0 = warp * per, q1 = min(tiles, q0 + per);
    int run = 0;
    if (i < kE)
#pragma unroll 16
        for (int q = q0; q < q1; ++q) run += h[(long long)q * kE];
    sum[warp][lane] = run;
    __syncthreads();
    run = 0;
    for (int w = 0; w < warp; ++w) run += sum[w][lane];
    if (i >= kE) return;
    for (int q = q0; q < q1; q += 16) {
        int v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = q + u < q1 ? h[(long long)(q + u) * kE] : 0;
#pragma unroll
        for (int u = 0; u < 16; ++u)
            if (q + u < q1) {
                h[(long long)(q + u) * kE] = run;
                run += v[u];
            }
    }
    if (warp == GT_WARPS - 1) all[(long long)t * kE + i] = run;
}

// SCANNED: behind gate_scan, for many tiles.
template <bool SCANNED>
__global__ void __launch_bounds__(GT_THREADS)
gate_slots_kernel(Dims p, int rows, const int32_t *__restrict__ idx, const int32_t *__restrict__ hist,
                  const int32_t *__restrict__ sums, int32_t *__restrict__ slot, int32_t *__restrict__ load,
                  int32_t *__restrict__ demand) {
    extern __shared__ int gt_base[];  // [k][E]: the next place of each (choice, expert); then [k][E] whole counts
    const int E = p.E, k = p.k, N = p.N, t = blockIdx.y, tiles = gridDim.x, tile = blockIdx.x;
    int *all = gt_base + k * E;
    pdl_wait();
    pdl_launch_dependents();
    const int32_t *h = hist + (long long)t * tiles * k * E;
    for (int i = threadIdx.x; i < k * E; i += GT_THREADS) {
        if (SCANNED) {
            gt_base[i] = h[(long long)tile * k * E + i];
            all[i] = sums[(long long)t * k * E + i];
            continue;
        }
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
    pdl_launch_dependents();
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

// Eight elements as they lie in memory.
template <typename T>
struct Row8 {
    uint4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
    }
    __device__ __forceinline__ void get(float *o) const {
        if constexpr (sizeof(T) == 2) {
            bf16x8_to_f32(v[0], o);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                o[4 * i] = __uint_as_float(v[i].x), o[4 * i + 1] = __uint_as_float(v[i].y);
                o[4 * i + 2] = __uint_as_float(v[i].z), o[4 * i + 3] = __uint_as_float(v[i].w);
            }
        }
    }
};

template <typename T, int KMAX>
__global__ void __launch_bounds__(GT_THREADS)
gate_grad_kernel(Dims p, Gating g, const float *__restrict__ logits, const int32_t *__restrict__ idx,
                 const float *__restrict__ gate, const int32_t *__restrict__ slot, const T *__restrict__ dy,
                 const T *__restrict__ ye, float *__restrict__ dgate, float *__restrict__ dlogits) {
    const int lane = threadIdx.x & 31, d = p.d, E = p.E, k = p.k;
    const long long tn = (long long)blockIdx.x * GT_WARPS + (threadIdx.x >> 5);
    pdl_wait();
    pdl_launch_dependents();
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
    float le[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) le[j] = g.score == VMOE_SCORE_SIGMOID && ei[j] >= 0 ? __ldg(logits + tn * E + ei[j]) : 0.0f;
    for (int v = lane * 8; v < d; v += 256) {  // a token's rows in flight together
        Row8<T> a, b[KMAX];
        a.load(dy + tn * d + v);
#pragma unroll
        for (int j = 0; j < KMAX; ++j)
            if (sl[j] >= 0) b[j].load(ye + (((long long)t * E + ei[j]) * p.C + sl[j]) * d + v);
        float fa[8];
        a.get(fa);
#pragma unroll
        for (int j = 0; j < KMAX; ++j) {
            if (sl[j] < 0) continue;
            float fb[8];
            b[j].get(fb);
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
        if (g.score == VMOE_SCORE_SIGMOID) c[j] *= 1.0f / (1.0f + expf(le[j]));
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

// Sums of K values over the warp, lane l < K getting the l-th's: in every step a lane gives half of its values away and adds
// up the other half's, 7 + 2 exchanges for eight values instead of 40.
template <int K>
__device__ __forceinline__ float sum_each(const float (&v)[K], int lane) {
    float h[K];
#pragma unroll
    for (int i = 0; i < K; ++i) h[i] = v[i];
    int o = 16;
#pragma unroll
    for (int n = K / 2; n > 0; n >>= 1, o >>= 1) {
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float give = up ? h[i] : h[i + n], keep = up ? h[i + n] : h[i];
            h[i] = keep + __shfl_xor_sync(FULL, give, o);
        }
    }
    float r = h[0];
    for (; o > 0; o >>= 1) r += __shfl_xor_sync(FULL, r, o);
    return __shfl_sync(FULL, r, lane * (32 / K) & 31);
}

// The same for more than four choices: lane j has choice j, the next token's ahead, four expert rows are in flight, and the
// sums are taken together.  80000 tokens, 6 of 30 experts, d 256: 85 us, the form above 134 (its 8 rows' registers 163).  With
// few choices this one's exchanges and its 60 registers cost more than they save: 8 x 1576 tokens, one of 64, d 1024: 19 us
// against 12; 8 x 2000, four of 32, d 768: 30 against 28.
template <typename T>
__global__ void __launch_bounds__(GT_THREADS, 4)
gate_grad_many_kernel(Dims p, Gating g, const float *__restrict__ logits, const int32_t *__restrict__ idx,
                      const float *__restrict__ gate, const int32_t *__restrict__ slot, const T *__restrict__ dy,
                      const T *__restrict__ ye, float *__restrict__ dgate, float *__restrict__ dlogits) {
    constexpr int KMAX = 8, U = 4;  // U expert rows in flight
    const int lane = threadIdx.x & 31, d = p.d, E = p.E, k = p.k;
    const long long TN = (long long)p.T * p.N, stride = (long long)gridDim.x * GT_WARPS;
    const bool add = (p.flags & VMOE_DLOGITS_ADD) != 0, dense = g.score == VMOE_SCORE_SOFTMAX && !g.renorm;
    pdl_wait();
    pdl_launch_dependents();
    // lane j: choice j's expert, slot and gate, the next token's ahead
    long long tn = (long long)blockIdx.x * GT_WARPS + (threadIdx.x >> 5);
    int e1 = -1, s1 = -1;
    float g1 = 0.0f;
    auto routing = [&](long long n) {
        e1 = s1 = -1;
        g1 = 0.0f;
        if (n < TN && lane < k) {
            e1 = __ldg(idx + n * k + lane);
            s1 = __ldg(slot + n * k + lane);
            g1 = __ldg(gate + n * k + lane);
        }
    };
    routing(tn);
    for (; tn < TN; tn += stride) {
        const int e = e1, sl = s1;
        const float gt = g1;
        const float *l = logits + tn * E;
        float *dl = dlogits + tn * E;
        float le = 0.0f;
        if (g.score == VMOE_SCORE_SIGMOID && e >= 0) le = __ldg(l + e);
        const T *yt = ye + (tn / p.N) * E * p.C * d;
        float dg[KMAX] = {};
        for (int v = lane * 8, v0 = 0; v0 < d; v += 256, v0 += 256) {
            Row8<T> a;
            if (v < d) a.load(dy + tn * d + v);
#pragma unroll
            for (int j0 = 0; j0 < KMAX; j0 += U) {
                if (j0 >= k) break;
                Row8<T> b[U];
                bool on[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int s = __shfl_sync(FULL, sl, j0 + u), ex = __shfl_sync(FULL, e, j0 + u);
                    on[u] = s >= 0 && v < d;
                    if (on[u]) b[u].load(yt + ((long long)ex * p.C + s) * d + v);
                }
                if (v0 == 0 && j0 == 0) routing(tn + stride);
                float fa[8];
                a.get(fa);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (!on[u]) continue;
                    float fb[8];
                    b[u].get(fb);
#pragma unroll
                    for (int q = 0; q < 8; ++q) dg[j0 + u] = fmaf(fa[q], fb[q], dg[j0 + u]);
                }
            }
        }
        const float mine = sum_each<KMAX>(dg, lane);
        // in the choices' order, as in gate_backward_scored: the two forms give the same values
        const float r = e >= 0 ? gt / g.scale : 0.0f;
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < KMAX; ++j) m = fmaf(__shfl_sync(FULL, r, j), __shfl_sync(FULL, mine, j), m);
        if (lane < k) dgate[tn * k + lane] = mine;
        if (dense && __any_sync(FULL, e >= 0)) {
            float mx = -INFINITY, sum = 0.0f;
            for (int i = lane; i < E; i += 32)
                if (fabsf(l[i]) < INFINITY) mx = fmaxf(mx, l[i]);
            mx = warp_max(mx);
            for (int i = lane; i < E; i += 32)
                if (fabsf(l[i]) < INFINITY) sum += expf(l[i] - mx);
            sum = warp_sum(sum);
            for (int i0 = 0; i0 < E; i0 += 32) {
                const int i = i0 + lane;
                float ge = 0.0f;
#pragma unroll
                for (int j = 0; j < KMAX; ++j) {
                    const int ej = __shfl_sync(FULL, e, j);
                    const float gj = __shfl_sync(FULL, mine, j);
                    if (ej == i) ge = gj;
                }
                if (i >= E) continue;
                float v = fabsf(l[i]) < INFINITY ? g.scale * (expf(l[i] - mx) / sum) * (ge - m) : 0.0f;
                if (add) v += dl[i];
                dl[i] = v;
            }
            continue;
        }
        // zeros, and the choices' values over them
        float c = e >= 0 ? gt * (g.renorm ? mine - m : mine) : 0.0f;
        if (g.score == VMOE_SCORE_SIGMOID) c *= 1.0f / (1.0f + expf(le));
        if (!add)
            for (int i = lane; i < E; i += 32) dl[i] = 0.0f;
        __syncwarp();
        if (e >= 0) dl[e] = add ? dl[e] + c : c;
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
    // four CTAs an SM, every warp several tokens
    const long long blocks = std::min(((long long)p.T * p.N + GT_WARPS - 1) / GT_WARPS, 4LL * num_sms());
    return launch_kernel(gate_grad_many_kernel<T>, dim3((unsigned)blocks), dim3(GT_THREADS), 0, s, p, g, logits, idx, gate,
                         slot, (const T *)dy, (const T *)ye, dgate, dlogits);
}

// Rows of a tile: 64, more where a task would have over 256 tiles (65536 x 4 rows of 256 experts: gate_fast 324 us with
// 128 tiles, 1.1 waves; 268 with 256; 260 with 512, and as much longer for their counts).
int tile_rows(int N) {
    int rows = 64;
    while (rows < 32768 && (N + rows - 1) / rows > 256) rows *= 2;  // their bits: 4 KB of shared memory
    return rows;
}

// Launch arguments of gate_rows and gate_fast.
struct RowArgs {
    Dims p;
    Gating g;
    int rows;
    const float *logits, *sbias;
    const uint8_t *mask;
    int32_t *idx;
    float *gate;
    int32_t *hist;
};
template <typename Kern>
int launch_rows(Kern kern, int M, const RowArgs &a, cudaStream_t s) {
    const size_t smem = row_scratch(M) + ((size_t)a.p.k * a.p.E + (a.rows + 31) / 32) * 4;
    return launch_kernel(kern, dim3((a.p.N + a.rows - 1) / a.rows, a.p.T), dim3(GT_THREADS), smem, s, a.p, a.g, a.rows, a.logits,
                         a.sbias, a.mask, a.idx, a.gate, a.hist);
}
int choose_rows(const RowArgs &a, cudaStream_t s) {
    const int E = a.p.E, gsize = E / a.g.groups;
    const int V = E > 128 ? 8 : 4;
    const bool aligned = a.g.groups == 1 || (gsize >= V && (gsize & (gsize - 1)) == 0);
    if (!aligned) {
        if (E <= 32) return launch_rows(gate_rows_kernel<1>, 1, a, s);
        if (E <= 64) return launch_rows(gate_rows_kernel<2>, 2, a, s);
        if (E <= 128) return launch_rows(gate_rows_kernel<4>, 4, a, s);
        return launch_rows(gate_rows_kernel<8>, 8, a, s);
    }
    int L = 1;  // lanes for the experts and for the choices
    while (L * V < E || L < a.p.k) L *= 2;
    if (V == 8) return launch_rows(gate_fast_kernel<32, 8>, 8, a, s);
    if (L <= 2) return launch_rows(gate_fast_kernel<2, 4>, 1, a, s);
    if (L <= 4) return launch_rows(gate_fast_kernel<4, 4>, 1, a, s);
    if (L <= 8) return launch_rows(gate_fast_kernel<8, 4>, 1, a, s);
    if (L <= 16) return launch_rows(gate_fast_kernel<16, 4>, 2, a, s);
    return launch_rows(gate_fast_kernel<32, 4>, 4, a, s);
}

}  // namespace

size_t gate_workspace(const Dims &p) {
    const int rows = tile_rows(p.N);
    return (size_t)p.T * ((p.N + rows - 1) / rows + 1) * p.k * p.E * 4;
}

int launch_gate(const Dims &p, const Gating &g, const float *logits, const float *sbias, const uint8_t *mask, int32_t *idx,
                float *gate, int32_t *slot, int32_t *load, int32_t *demand, int32_t *hist, cudaStream_t s) {
    const int rows = tile_rows(p.N), tiles = (p.N + rows - 1) / rows, kE = p.k * p.E;
    trace_before(s, "gate_rows");
    int st = choose_rows(RowArgs{p, g, rows, logits, sbias, mask, idx, gate, hist}, s);
    trace_after(s);
    if (st != VMOE_OK) return st;
    int32_t *all = hist + (long long)p.T * tiles * kE;
    const bool scan = tiles > 32;
    if (scan) {
        trace_before(s, "gate_scan");
        st = launch_kernel(gate_scan_kernel, dim3((kE + 31) / 32, p.T), dim3(GT_THREADS), 0, s, kE, tiles,
                           hist, all);
        trace_after(s);
        if (st != VMOE_OK) return st;
    }
    trace_before(s, "gate_slots");
    st = launch_kernel(scan ? gate_slots_kernel<true> : gate_slots_kernel<false>, dim3(tiles, p.T), dim3(GT_THREADS),
                       (size_t)kE * 8, s, p, rows, idx, hist, all, slot, load, demand);
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

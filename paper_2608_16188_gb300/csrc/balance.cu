// balance.cu -- the routers' balance losses with per-expert counts, and their
// gradient into the logits (the capacity limits of Challenge #1 drop what an
// uneven router sends to a full expert; these losses keep the load even).
//
// With p = softmax(logits) and M the tokens of a task that take part:
//   count_e  = choices of expert e, before capacity drops any
//   excess_e = sum_n p_e - M / E
//   loss 0   = E / (k M^2) sum_e count_e sum_n p_e
//   loss 1   = E / M^2 sum_e excess_e^2            (squared variation of the importances)
//   loss 2   = 1 / M sum_n lse_n^2                 (lse = log sum_e exp(logit))
// Their gradient by p does not depend on the token, so one coefficient an expert
// carries it: dlogit_e = p_e (c_e - sum_i p_i c_i + z lse).
//
// A row of E logits lies in the registers of L neighbouring lanes, V to a lane, and is
// read once; L is the smallest power of two that holds it, and a lane works on R rows
// at a time, with the next R rows' loads in flight.  exp(x - max) is taken with the row's
// maximum, of R rows in one butterfly.  (Less the row's first logit, which needs no maximum,
// the exponents of a row whose first expert is far below the others reach 100, where half
// a step is 4e-6, and lse = c + log(sum) cancels.)  The importances are summed less their
// even share, so that what is left after M / E cancels keeps its bits, in runs of SUM_RUN rows a
// thread, then over the runs.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "around.cuh"

namespace cg = cooperative_groups;

namespace vmoe {

namespace {

constexpr int BT = 256;      // threads a CTA
constexpr int R = 4;         // rows a lane works on at a time
constexpr int SUM_RUN = 16;  // steps of R rows a thread sums before it adds them to its total
constexpr int CLUSTER = 8;   // CTAs that join their sums through distributed shared memory
// Steps of a CTA of a cluster before two launches are faster.  On the GPU 16 steps in all
// took 4.9 to 5.5 us as a cluster of eight and 5.8 to 6.5 in two launches, 32 steps 6.7 to
// 7.7 and 6.3 to 6.7 (one and eight tasks, 32 and 256 experts), 64 steps 10.1 to 11.6 and
// 6.4 to 8.2; the second launch costs the host 1.9 us.
constexpr int JOIN_STEPS = 4;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

int lanes_of(int E) {
    int L = 1;
    while (L < 32 && 4 * L < E) L *= 2;
    return L;
}
int rows_of(const Dims &p) { return BT / lanes_of(p.E) * R; }  // a CTA's rows at a time

// CTAs that fill the card once: two an SM above 128 experts (108 to 128 registers), three
// below.
int ctas_of(const Dims &p) { return 152 * (p.E > 128 ? 2 : 3); }

// Slices of the tokens of a task, a CTA each.  Up to CLUSTER of them are a cluster, which
// joins its sums itself; more leave them in the workspace for a second launch.
int slices_of(const Dims &p) {
    const int steps = (p.N + rows_of(p) - 1) / rows_of(p);
    if (steps <= CLUSTER * JOIN_STEPS) {
        int n = 1;
        while (n < CLUSTER && n < steps) n *= 2;
        return n;
    }
    return std::max(CLUSTER, std::min(steps, ctas_of(p) / p.T));
}
bool two_launches(const Dims &p) { return slices_of(p) > CLUSTER; }

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float lg2(float v) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Totals of Q values over the L lanes of a row, the same in all of them.  While lanes and
// values last, a step of the butterfly sums two values at once.
template <int L, int Q>
__device__ __forceinline__ void row_totals(float (&v)[Q]) {
    if constexpr (L < Q) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < Q; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    } else {
        const int lane = threadIdx.x % L;
#pragma unroll
        for (int h = Q / 2, o = L / 2; h > 0; h >>= 1, o >>= 1) {
            const bool up = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < h; ++i) {
                const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        }
#pragma unroll
        for (int o = L / Q / 2; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        const float sum = v[0];
#pragma unroll
        for (int i = 0; i < Q; ++i) v[i] = __shfl_sync(0xffffffffu, sum, i * (L / Q), L);
    }
}
// The same for maxima (a NaN is passed over).
template <int L, int Q>
__device__ __forceinline__ void row_maxima(float (&v)[Q]) {
    if constexpr (L < Q) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < Q; ++i) v[i] = fmaxf(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
    } else {
        const int lane = threadIdx.x % L;
#pragma unroll
        for (int h = Q / 2, o = L / 2; h > 0; h >>= 1, o >>= 1) {
            const bool up = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < h; ++i) {
                const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
                v[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, o));
            }
        }
#pragma unroll
        for (int o = L / Q / 2; o > 0; o >>= 1) v[0] = fmaxf(v[0], __shfl_xor_sync(0xffffffffu, v[0], o));
        const float top = v[0];
#pragma unroll
        for (int i = 0; i < Q; ++i) v[i] = __shfl_sync(0xffffffffu, top, i * (L / Q), L);
    }
}

// Column of a lane's value i: runs of four, one after the other over the lanes.
template <int L>
__device__ __forceinline__ int column(int lane, int i) { return (i >> 2) * 4 * L + 4 * lane + (i & 3); }

// A lane's V values of a row, as pairs; -inf behind the last expert, 0 everywhere where
// the row is not to be read.
template <int L, int V, bool VEC>
__device__ __forceinline__ void load_row(const float *row, int E, int lane, bool in, f32x2 (&x)[V / 2]) {
    const float none = in ? -INFINITY : 0.0f;
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        const int c = column<L>(lane, j);
        if (VEC) {
            x[j / 2] = x[j / 2 + 1] = pk2(none);
            if (in && c < E) {
                const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(row + c);
                x[j / 2] = v.x;
                x[j / 2 + 1] = v.y;
            }
        } else {
            float f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = in && c + i < E ? row[c + i] : none;
            x[j / 2] = pk2(f[0], f[1]);
            x[j / 2 + 1] = pk2(f[2], f[3]);
        }
    }
}

// x[r] becomes exp(x[r] - c[r]), c[r] the row's maximum (0 where that is -inf: nowhere to
// go, a sum of 0; NaN and +inf make the sum NaN).
template <int L, int V>
__device__ __forceinline__ void exp_rows(f32x2 (&x)[R][V / 2], float (&c)[R], float (&sum)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
        c[r] = -INFINITY;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) c[r] = fmaxf(c[r], fmaxf(unpk2(x[r][i]).x, unpk2(x[r][i]).y));
    }
    row_maxima<L, R>(c);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (c[r] == -INFINITY) c[r] = 0.0f;
        const f32x2 mc = pk2(-c[r]);
        f32x2 s = 0;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 a = unpk2(mul2(add2(x[r][i], mc), pk2(LOG2E)));
            x[r][i] = pk2(ex2(a.x), ex2(a.y));
            s = add2(s, x[r][i]);
        }
        const float2 two = unpk2(s);
        sum[r] = two.x + two.y;
    }
    row_totals<L, R>(sum);
}

// A CTA's sums.
struct Sums {
    float excess[256];
    int count[256];
    float lse;
    int tokens;
};
__host__ __device__ inline int part_words(int E) { return 2 * E + 2; }

// Totals of three values over the CTA, in thread 0.
__device__ __forceinline__ float3 block_sum(float3 v) {
    __shared__ float3 buf[32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
        v.z += __shfl_xor_sync(0xffffffffu, v.z, o);
    }
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    float3 s = make_float3(0.0f, 0.0f, 0.0f);
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {
            s.x += buf[w].x;
            s.y += buf[w].y;
            s.z += buf[w].z;
        }
    return s;
}

struct Out {
    int32_t *count, *tokens;
    float *excess, *loss;
};

// The cluster's sums joined in rank order by its first CTA, and the losses.
__device__ __forceinline__ void finish(Sums &mine, const Dims &p, int t, const Out &o) {
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks();
    cluster.sync();
    if (cluster.block_rank() == 0) {
        const int e = threadIdx.x, E = p.E;
        float3 part = make_float3(0.0f, 0.0f, 0.0f);
        if (e < E) {
            float v = 0.0f;
            int c = 0;
            for (int q = 0; q < ranks; ++q) {
                const Sums *s = cluster.map_shared_rank(&mine, q);
                v += s->excess[e];
                c += s->count[e];
            }
            o.count[(long long)t * E + e] = c;
            o.excess[(long long)t * E + e] = v;
            part = make_float3((float)c * v, v * v, (float)c);
        }
        part = block_sum(part);
        if (threadIdx.x == 0) {
            float l = 0.0f;
            int m = 0;
            for (int q = 0; q < ranks; ++q) {
                const Sums *s = cluster.map_shared_rank(&mine, q);
                l += s->lse;
                m += s->tokens;
            }
            const float M = (float)max(m, 1), fe = (float)E, km = (float)p.k * M;
            o.tokens[t] = m;
            o.loss[3LL * t] = m ? part.z / km + part.x * (fe / km) / M : 0.0f;
            o.loss[3LL * t + 1] = m ? part.y * (fe / M) / M : 0.0f;
            o.loss[3LL * t + 2] = m ? l / M : 0.0f;
        }
    }
    cluster.sync();  // the sums stay until they are read
}

// grid (slices, T): the sums of a slice of a task's tokens, joined by the cluster or
// left in `parts`.
template <int L, int V, bool VEC>
__global__ void __launch_bounds__(BT)
balance_kernel(Dims p, const float *__restrict__ logits, const int32_t *__restrict__ idx,
               const uint8_t *__restrict__ mask, float *__restrict__ parts, Out o) {
    __shared__ Sums sums;
    __shared__ float warp_sums[BT / 32][4 * L * (V / 4)];
    __shared__ float warp_lse[BT / 32];
    __shared__ int warp_tokens[BT / 32];
    constexpr int G = 32 / L;  // groups of lanes, R rows each, in a warp
    const int tid = threadIdx.x, warp = tid >> 5, wl = tid & 31, lane = wl % L, group = wl / L;
    const int t = blockIdx.y, N = p.N, E = p.E, k = p.k;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    pdl_wait();
    for (int e = tid; e < E; e += BT) sums.count[e] = 0;
    __syncthreads();
    const float *lt = logits + (long long)t * N * E;
    const int32_t *it = idx + (long long)t * N * k;
    const uint8_t *mt = mask ? mask + (long long)t * N : nullptr;
    const float even = 1.0f / (float)E;
    f32x2 total[V / 2] = {};
    float lse_total = 0.0f;
    int tokens = 0;
    f32x2 next[R][V / 2];
    unsigned next_in = 0;
    int next_e = -1;  // a lane's first of the choices of those rows, which lie one after the other
    auto fetch = [&](int n0) {  // the warp's G x R rows from n0 on
        next_in = 0;
        next_e = wl < min(G * R, end - n0) * k ? it[(long long)n0 * k + wl] : -1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = n0 + group * R + r;
            const bool in = n < end && (!mt || mt[n] != 0);
            next_in |= (unsigned)in << r;
            load_row<L, V, VEC>(lt + (long long)n * E, E, lane, in, next[r]);
        }
    };
    constexpr int STEP = BT / 32 * G * R;
    const int first = beg + warp * G * R;
    fetch(first);
    // every lane of a warp walks the same steps: the shuffles need them all
    for (int n0 = first; n0 < end;) {
        f32x2 run[V / 2] = {};
        float lse_run = 0.0f;
        int live_rows = 0;
        for (int i = 0; i < SUM_RUN && n0 < end; ++i, n0 += STEP) {
            f32x2 x[R][V / 2];
            unsigned live = next_in;
            int e = next_e;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < V / 2; ++j) x[r][j] = next[r][j];
            if (n0 + STEP < end) fetch(n0 + STEP);
            float c[R], s[R];
            exp_rows<L, V>(x, c, s);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (s[r] == 0.0f) live &= ~(1u << r);
                const bool on = (live >> r & 1) != 0;
                const f32x2 inv = pk2(on ? rcp(s[r]) : 0.0f);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) run[j] = fma2(x[r][j], inv, run[j]);
                const float lse = fmaf(lg2(s[r]), LN2, c[r]);
                if (on) lse_run = fmaf(lse, lse, lse_run);
            }
            live_rows += __popc(live);
            const int choices = G * R * k;
            const int32_t *ip = it + (long long)n0 * k;
            for (int j = wl; j - wl < choices; j += 32) {
                const int row = j / k;
                const unsigned bits = __shfl_sync(0xffffffffu, live, min(row / R, G - 1) * L);
                if (j < choices && (bits >> (row % R) & 1)) {
                    if (j >= 32) e = ip[j];
                    if ((unsigned)e < (unsigned)E) atomicAdd(&sums.count[e], 1);
                }
            }
        }
        tokens += live_rows;
        lse_total += lse_run;
        const f32x2 share = pk2(-(float)live_rows * even);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) total[j] = add2(total[j], add2(run[j], share));
    }
    // the rows of a warp, then of the CTA
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 two = unpk2(total[j / 2]);
        float v = j & 1 ? two.y : two.x;
#pragma unroll
        for (int o2 = L; o2 < 32; o2 <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o2);
        if (wl < L) warp_sums[warp][column<L>(lane, j)] = v;
    }
#pragma unroll
    for (int o2 = L; o2 < 32; o2 <<= 1) {
        lse_total += __shfl_xor_sync(0xffffffffu, lse_total, o2);
        tokens += __shfl_xor_sync(0xffffffffu, tokens, o2);
    }
    if (wl == 0) {
        warp_lse[warp] = lse_total;
        warp_tokens[warp] = tokens;
    }
    __syncthreads();
    if (tid < E) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < BT / 32; ++w) v += warp_sums[w][tid];
        sums.excess[tid] = v;
    }
    if (tid == 0) {
        float v = 0.0f;
        int n = 0;
#pragma unroll
        for (int w = 0; w < BT / 32; ++w) {
            v += warp_lse[w];
            n += warp_tokens[w];
        }
        sums.lse = v;
        sums.tokens = n;
    }
    if (parts == nullptr) {
        finish(sums, p, t, o);
        return;
    }
    __syncthreads();
    float *out = parts + ((long long)t * gridDim.x + blockIdx.x) * part_words(E);
    if (tid < E) {
        out[tid] = sums.excess[tid];
        out[E + tid] = __int_as_float(sums.count[tid]);
    }
    if (tid == 0) {
        out[2 * E] = sums.lse;
        out[2 * E + 1] = __int_as_float(sums.tokens);
    }
}

constexpr int FT = 1024;  // threads of the last sum: 4 runs of the parts for each of 256 experts

// grid (CLUSTER, T), a cluster a task: the slices' sums joined, in their order.
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(FT)
balance_join_kernel(Dims p, int slices, const float *__restrict__ parts, Out o) {
    __shared__ Sums sums;
    __shared__ float ex[4][256];
    __shared__ int cn[4][256];
    const int tid = threadIdx.x, t = blockIdx.y, E = p.E, e = tid & 255, q = tid >> 8;
    const int lo = slices * (int)blockIdx.x / CLUSTER, hi = slices * ((int)blockIdx.x + 1) / CLUSTER;
    pdl_wait();
    const float *in = parts + (long long)t * slices * part_words(E);
    const int beg = lo + (hi - lo) * q / 4, end = lo + (hi - lo) * (q + 1) / 4;
    float v = 0.0f;
    int c = 0;
    if (e < E)
        for (int i = beg; i < end; ++i) {
            v += in[(long long)i * part_words(E) + e];
            c += __float_as_int(in[(long long)i * part_words(E) + E + e]);
        }
    ex[q][e] = v;
    cn[q][e] = c;
    if (tid < 32) {
        float l = 0.0f;
        int m = 0;
        for (int i = lo + tid; i < hi; i += 32) {
            l += in[(long long)i * part_words(E) + 2 * E];
            m += __float_as_int(in[(long long)i * part_words(E) + 2 * E + 1]);
        }
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, s);
            m += __shfl_xor_sync(0xffffffffu, m, s);
        }
        if (tid == 0) {
            sums.lse = l;
            sums.tokens = m;
        }
    }
    __syncthreads();
    if (tid < 256) {
        sums.excess[tid] = (ex[0][tid] + ex[1][tid]) + (ex[2][tid] + ex[3][tid]);
        sums.count[tid] = (cn[0][tid] + cn[1][tid]) + (cn[2][tid] + cn[3][tid]);
    }
    finish(sums, p, t, o);
}

// grid (slices, T): dlogits of a slice of a task's tokens.
template <int L, int V, bool VEC>
__global__ void __launch_bounds__(BT)
balance_bwd_kernel(Dims p, const float *logits, const uint8_t *__restrict__ mask, const int32_t *__restrict__ count,
                   const int32_t *__restrict__ tokens, const float *__restrict__ excess, const float *__restrict__ dloss,
                   float *dlogits) {
    constexpr int G = 32 / L, STEP = BT / 32 * G * R;
    const int tid = threadIdx.x, wl = tid & 31, lane = wl % L, group = wl / L;
    const int t = blockIdx.y, N = p.N, E = p.E;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    pdl_wait();
    const float *lt = logits + (long long)t * N * E;
    float *dt = dlogits + (long long)t * N * E;
    const uint8_t *mt = mask ? mask + (long long)t * N : nullptr;
    f32x2 next[R][V / 2];
    unsigned next_in = 0;
    auto fetch = [&](int n0) {
        next_in = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = n0 + group * R + r;
            const bool in = n < end && (!mt || mt[n] != 0);
            next_in |= (unsigned)in << r;
            load_row<L, V, VEC>(lt + (long long)n * E, E, lane, in, next[r]);
        }
    };
    const int first = beg + (tid >> 5) * G * R;
    fetch(first);
    const float M = (float)max(tokens[t], 1), fe = (float)E;
    const float a0 = dloss[3 * t] * (fe / ((float)p.k * M)) / M, a1 = dloss[3 * t + 1] * (2.0f * fe / M) / M;
    const float z = dloss[3 * t + 2] * 2.0f / M;
    // any constant taken off the counts cancels in c - sum p c: their mean, so that little does
    f32x2 c[V / 2];
    {
        float n[V], all[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = column<L>(lane, i);
            n[i] = e < E ? (float)count[(long long)t * E + e] : 0.0f;
            all[0] += n[i];
        }
        row_totals<L, 1>(all);
        all[0] /= fe;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = column<L>(lane, i);
            n[i] = e < E ? a0 * (n[i] - all[0]) + a1 * excess[(long long)t * E + e] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) c[i] = pk2(n[2 * i], n[2 * i + 1]);
    }
    for (int n0 = first; n0 < end; n0 += STEP) {
        f32x2 x[R][V / 2];
        const unsigned in = next_in;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < V / 2; ++j) x[r][j] = next[r][j];
        if (n0 + STEP < end) fetch(n0 + STEP);
        float base[R], s[R], mean[R];
        exp_rows<L, V>(x, base, s);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2 m = 0;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) m = fma2(x[r][j], c[j], m);
            const float2 two = unpk2(m);
            mean[r] = two.x + two.y;
        }
        row_totals<L, R>(mean);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = n0 + group * R + r;
            const float inv = (in >> r & 1) && s[r] != 0.0f ? rcp(s[r]) : 0.0f;
            const f32x2 add = pk2(inv == 0.0f ? 0.0f : fmaf(z, fmaf(lg2(s[r]), LN2, base[r]), -mean[r] * inv));
            if (n >= end) continue;
            float *out = dt + (long long)n * E;
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const int e = column<L>(lane, j);
                // 0 for a token that does not take part, also where c is no number
                const f32x2 lo = inv == 0.0f ? 0 : mul2(mul2(x[r][j / 2], pk2(inv)), add2(c[j / 2], add));
                const f32x2 hi = inv == 0.0f ? 0 : mul2(mul2(x[r][j / 2 + 1], pk2(inv)), add2(c[j / 2 + 1], add));
                if (VEC) {
                    if (e < E) *reinterpret_cast<ulonglong2 *>(out + e) = make_ulonglong2(lo, hi);
                } else {
                    const float2 f = unpk2(lo), g = unpk2(hi);
                    if (e < E) out[e] = f.x;
                    if (e + 1 < E) out[e + 1] = f.y;
                    if (e + 2 < E) out[e + 2] = g.x;
                    if (e + 3 < E) out[e + 3] = g.y;
                }
            }
        }
    }
}

// Calls f(L, V, VEC) as constants for a problem of E experts.
template <int I>
using Int = std::integral_constant<int, I>;
template <typename F>
int with_layout(int E, F f) {
    auto vec = [&](auto L, auto V) {
        return E % 4 == 0 ? f(L, V, std::true_type()) : f(L, V, std::false_type());
    };
    if (E > 128) return vec(Int<32>(), Int<8>());
    switch (lanes_of(E)) {
        case 1: return vec(Int<1>(), Int<4>());
        case 2: return vec(Int<2>(), Int<4>());
        case 4: return vec(Int<4>(), Int<4>());
        case 8: return vec(Int<8>(), Int<4>());
        case 16: return vec(Int<16>(), Int<4>());
        default: return vec(Int<32>(), Int<4>());
    }
}

}  // namespace

size_t balance_workspace(const Dims &p) {
    return two_launches(p) ? (size_t)p.T * slices_of(p) * part_words(p.E) * sizeof(float) : 16;
}

int launch_balance(const Dims &p, const float *logits, const int32_t *idx, const uint8_t *mask, int32_t *count,
                   int32_t *tokens, float *excess, float *loss, float *parts, cudaStream_t s) {
    const int slices = slices_of(p);
    const bool two = two_launches(p);
    const Out o = {count, tokens, excess, loss};
    trace_before(s, "balance");
    int st = with_layout(p.E, [&](auto L, auto V, auto vec) {
        auto kern = balance_kernel<L(), V(), vec()>;
        if (two) return launch_kernel(kern, dim3(slices, p.T), dim3(BT), 0, s, p, logits, idx, mask, parts, o);
        return launch_cluster(kern, dim3(slices, p.T), dim3(BT), 0, slices, s, p, logits, idx, mask, (float *)nullptr, o);
    });
    trace_after(s);
    if (st != VMOE_OK || !two) return st;
    trace_before(s, "balance_join");
    st = launch_kernel(balance_join_kernel, dim3(CLUSTER, p.T), dim3(FT), 0, s, p, slices, (const float *)parts, o);
    trace_after(s);
    return st;
}

int launch_balance_bwd(const Dims &p, const float *logits, const uint8_t *mask, const int32_t *count,
                       const int32_t *tokens, const float *excess, const float *dloss, float *dlogits, cudaStream_t s) {
    const int steps = (p.N + rows_of(p) - 1) / rows_of(p), slices = std::max(1, std::min(steps, ctas_of(p) / p.T));
    trace_before(s, "balance_bwd");
    const int st = with_layout(p.E, [&](auto L, auto V, auto vec) {
        return launch_kernel(balance_bwd_kernel<L(), V(), vec()>, dim3(slices, p.T), dim3(BT), 0, s, p, logits,
                             mask, count, tokens, excess, dloss, dlogits);
    });
    trace_after(s);
    return st;
}

}  // namespace vmoe

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
// A row of E logits lies in the registers of L neighbouring lanes, V to a lane,
// and is read once; L is the smallest power of two that holds it.  The importances
// are summed less their even share, so that what is left after M / E cancels keeps
// its bits, in runs of SUM_RUN rows a thread, then over the runs.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"

namespace vmoe {

namespace {

constexpr int BT = 256;       // threads a CTA
constexpr int SUM_RUN = 32;   // rows a thread sums before it adds them to its total
constexpr int CTAS = 608;     // CTAs aimed at: 152 SMs x 4

// A CTA's sums, in fp32 words: excess[E], count[E] (int32), lse^2, tokens (int32).
__host__ __device__ inline int part_words(int E) { return 2 * E + 2; }

int lanes_of(int E) {
    int L = 1;
    while (L < 32 && 4 * L < E) L *= 2;
    return L;
}
// Slices of the tokens of a task, a CTA each.
int chunks_of(const Dims &p) {
    const int rows = BT / lanes_of(p.E);
    const int most = (p.N + 4 * rows - 1) / (4 * rows);
    return std::max(1, std::min(most, (CTAS + p.T - 1) / p.T));
}

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

template <int L>
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int L>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Column of a lane's value i: runs of four, one after the other over the lanes.
template <int L>
__device__ __forceinline__ int column(int lane, int i) { return (i >> 2) * 4 * L + 4 * lane + (i & 3); }

template <int L, int V, bool VEC>
__device__ __forceinline__ void load_row(const float *row, int E, int lane, float (&x)[V]) {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        const int c = column<L>(lane, j);
        if (VEC) {
            float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (c < E) v = __ldg(reinterpret_cast<const float4 *>(row + c));
            x[j] = v.x; x[j + 1] = v.y; x[j + 2] = v.z; x[j + 3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[j + i] = c + i < E ? __ldg(row + c + i) : -INFINITY;
        }
    }
}

// x becomes exp(x - max); returns the row's sum (0 when every logit is -inf: such a
// token takes no part) and its maximum.  A NaN or +inf makes the sum NaN.
template <int L, int V>
__device__ __forceinline__ float exp_row(float (&x)[V], float &top) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) m = fmaxf(m, x[i]);
    m = row_max<L>(m);
    if (m == -INFINITY) m = 0.0f;
    top = m;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = ex2((x[i] - m) * 1.4426950408889634f);
        s += x[i];
    }
    return row_sum<L>(s);
}

// grid (chunks, T): the sums of a slice of a task's tokens.
template <int L, int V, bool VEC>
__global__ void __launch_bounds__(BT)
balance_kernel(Dims p, const float *__restrict__ logits, const int32_t *__restrict__ idx,
               const uint8_t *__restrict__ mask, float *__restrict__ parts) {
    __shared__ float sums[BT / 32][256];
    __shared__ int hist[256];
    __shared__ float lse_sum[BT / 32];
    __shared__ int tok_sum[BT / 32];
    constexpr int R = BT / L;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid % L, group = tid / L;
    const int t = blockIdx.y, N = p.N, E = p.E, k = p.k;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    pdl_wait();
    for (int e = tid; e < E; e += BT) hist[e] = 0;
    __syncthreads();
    const float *lt = logits + (long long)t * N * E;
    const int32_t *it = idx + (long long)t * N * k;
    const uint8_t *mt = mask ? mask + (long long)t * N : nullptr;
    const float even = 1.0f / (float)E;
    float total[V] = {}, lse_total = 0.0f;
    int tokens = 0;
    // every lane of a warp walks the same number of rows: the shuffles need them all
    for (int n0 = beg; n0 < end; n0 += R * SUM_RUN) {
        float run[V] = {}, lse_run = 0.0f;
        int live_rows = 0;
        const int stop = min(end, n0 + R * SUM_RUN);
        for (int b = n0; b < stop; b += R) {
            const int n = b + group;
            const bool in = n < stop && (!mt || mt[n] != 0);
            float x[V], top;
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = -INFINITY;
            if (in) load_row<L, V, VEC>(lt + (long long)n * E, E, lane, x);
            const float s = exp_row<L, V>(x, top);
            if (s == 0.0f) continue;
            const float inv = 1.0f / s;
#pragma unroll
            for (int i = 0; i < V; ++i) run[i] = fmaf(x[i], inv, run[i]);
            ++live_rows;
            for (int j = lane; j < k; j += L) {
                const int e = __ldg(it + (long long)n * k + j);
                if ((unsigned)e < (unsigned)E) atomicAdd(&hist[e], 1);
            }
            const float lse = top + logf(s);
            lse_run = fmaf(lse, lse, lse_run);
        }
        tokens += live_rows;
        lse_total += lse_run;
#pragma unroll
        for (int i = 0; i < V; ++i) total[i] += run[i] - (float)live_rows * even;
    }
    // the rows of a warp, then of the CTA
#pragma unroll
    for (int o = L; o < 32; o <<= 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) total[i] += __shfl_xor_sync(0xffffffffu, total[i], o);
        lse_total += __shfl_xor_sync(0xffffffffu, lse_total, o);
        tokens += __shfl_xor_sync(0xffffffffu, tokens, o);
    }
    if ((tid & 31) < L) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (column<L>(lane, i) < E) sums[warp][column<L>(lane, i)] = total[i];
    }
    if ((tid & 31) == 0) {
        lse_sum[warp] = lse_total;
        tok_sum[warp] = tokens;
    }
    __syncthreads();
    float *out = parts + ((long long)t * gridDim.x + blockIdx.x) * part_words(E);
    for (int e = tid; e < E; e += BT) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < BT / 32; ++w) v += sums[w][e];
        out[e] = v;
        out[E + e] = __int_as_float(hist[e]);
    }
    if (tid == 0) {
        float v = 0.0f;
        int n = 0;
#pragma unroll
        for (int w = 0; w < BT / 32; ++w) {
            v += lse_sum[w];
            n += tok_sum[w];
        }
        out[2 * E] = v;
        out[2 * E + 1] = __int_as_float(n);
    }
}

constexpr int FT = 1024;  // threads of the last sum: 4 slices of the parts for each of 256 experts

__device__ __forceinline__ float block_sum(float v, float *buf) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (int)threadIdx.x < (int)(blockDim.x >> 5) ? buf[threadIdx.x] : 0.0f;
    if (threadIdx.x < 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    }
    return v;  // in thread 0
}

// grid (T): the slices' sums joined, in their order, and the losses.
__global__ void __launch_bounds__(FT)
balance_join_kernel(Dims p, int chunks, const float *__restrict__ parts, int32_t *__restrict__ count,
                    int32_t *__restrict__ tokens, float *__restrict__ excess, float *__restrict__ loss) {
    __shared__ float ex[4][256];
    __shared__ int cn[4][256];
    __shared__ float buf[FT / 32];
    const int tid = threadIdx.x, t = blockIdx.x, E = p.E, e = tid & 255, q = tid >> 8;
    pdl_wait();
    const float *in = parts + (long long)t * chunks * part_words(E);
    const int beg = chunks * q / 4, end = chunks * (q + 1) / 4;
    float v = 0.0f;
    int c = 0;
    if (e < E)
        for (int i = beg; i < end; ++i) {
            v += in[(long long)i * part_words(E) + e];
            c += __float_as_int(in[(long long)i * part_words(E) + E + e]);
        }
    ex[q][e] = v;
    cn[q][e] = c;
    float l = 0.0f;
    int m = 0;
    for (int i = tid; i < chunks; i += FT) {
        l += in[(long long)i * part_words(E) + 2 * E];
        m += __float_as_int(in[(long long)i * part_words(E) + 2 * E + 1]);
    }
    l = block_sum(l, buf);
    __syncthreads();
    int *ibuf = reinterpret_cast<int *>(buf);
    m = __reduce_add_sync(0xffffffffu, m);
    if ((tid & 31) == 0) ibuf[tid >> 5] = m;
    __syncthreads();
    m = 0;
    for (int w = 0; w < FT / 32; ++w) m += ibuf[w];
    float both = 0.0f, square = 0.0f, all = 0.0f;
    if (tid < E) {
        v = (ex[0][e] + ex[1][e]) + (ex[2][e] + ex[3][e]);
        c = (cn[0][e] + cn[1][e]) + (cn[2][e] + cn[3][e]);
        count[(long long)t * E + e] = c;
        excess[(long long)t * E + e] = v;
        both = (float)c * v;
        square = v * v;
        all = (float)c;
    }
    both = block_sum(both, buf);
    square = block_sum(square, buf);
    all = block_sum(all, buf);
    if (tid == 0) {
        const float M = (float)max(m, 1), fe = (float)E, km = (float)p.k * M;
        tokens[t] = m;
        float *out = loss + 3LL * t;
        out[0] = m ? all / km + both * (fe / km) / M : 0.0f;
        out[1] = m ? square * (fe / M) / M : 0.0f;
        out[2] = m ? l / M : 0.0f;
    }
}

// grid (chunks, T): dlogits of a slice of a task's tokens.
template <int L, int V, bool VEC>
__global__ void __launch_bounds__(BT)
balance_bwd_kernel(Dims p, const float *__restrict__ logits, const uint8_t *__restrict__ mask,
                   const int32_t *__restrict__ count, const int32_t *__restrict__ tokens,
                   const float *__restrict__ excess, const float *__restrict__ dloss, float *__restrict__ dlogits) {
    constexpr int R = BT / L;
    const int tid = threadIdx.x, lane = tid % L, group = tid / L;
    const int t = blockIdx.y, N = p.N, E = p.E;
    const int beg = (int)((long long)N * blockIdx.x / gridDim.x), end = (int)((long long)N * (blockIdx.x + 1) / gridDim.x);
    pdl_wait();
    const float M = (float)max(tokens[t], 1), fe = (float)E;
    const float a0 = dloss[3 * t] * (fe / ((float)p.k * M)) / M, a1 = dloss[3 * t + 1] * (2.0f * fe / M) / M;
    const float z = dloss[3 * t + 2] * 2.0f / M;
    // any constant taken off the counts cancels in c - sum p c: their mean, so that little does
    float c[V], all = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = column<L>(lane, i);
        c[i] = e < E ? (float)count[(long long)t * E + e] : 0.0f;
        all += c[i];
    }
    all = row_sum<L>(all) / fe;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = column<L>(lane, i);
        c[i] = e < E ? a0 * (c[i] - all) + a1 * excess[(long long)t * E + e] : 0.0f;
    }
    const float *lt = logits + (long long)t * N * E;
    float *dt = dlogits + (long long)t * N * E;
    const uint8_t *mt = mask ? mask + (long long)t * N : nullptr;
    for (int b = beg; b < end; b += R) {
        const int n = b + group;
        const bool row = n < end, in = row && (!mt || mt[n] != 0);
        float x[V], top;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = -INFINITY;
        if (in) load_row<L, V, VEC>(lt + (long long)n * E, E, lane, x);
        const float s = exp_row<L, V>(x, top);
        const float inv = s == 0.0f ? 0.0f : 1.0f / s;
        float mean = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] *= inv;
            mean = fmaf(x[i], c[i], mean);
        }
        mean = row_sum<L>(mean);
        const float add = s == 0.0f ? 0.0f : fmaf(z, top + logf(s), -mean);
        if (!row) continue;
        float *out = dt + (long long)n * E;
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const int e = column<L>(lane, j);
            const float r0 = x[j] * (c[j] + add), r1 = x[j + 1] * (c[j + 1] + add);
            const float r2 = x[j + 2] * (c[j + 2] + add), r3 = x[j + 3] * (c[j + 3] + add);
            if (VEC) {
                if (e < E) *reinterpret_cast<float4 *>(out + e) = make_float4(r0, r1, r2, r3);
            } else {
                if (e < E) out[e] = r0;
                if (e + 1 < E) out[e + 1] = r1;
                if (e + 2 < E) out[e + 2] = r2;
                if (e + 3 < E) out[e + 3] = r3;
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

size_t balance_workspace(const Dims &p) { return (size_t)p.T * chunks_of(p) * part_words(p.E) * sizeof(float); }

int launch_balance(const Dims &p, const float *logits, const int32_t *idx, const uint8_t *mask, int32_t *count,
                   int32_t *tokens, float *excess, float *loss, float *parts, cudaStream_t s) {
    const int chunks = chunks_of(p);
    trace_before(s, "balance");
    int st = with_layout(p.E, [&](auto L, auto V, auto vec) {
        return launch_kernel(balance_kernel<L(), V(), vec()>, dim3(chunks, p.T), dim3(BT), 0, s, p, logits, idx, mask, parts);
    });
    trace_after(s);
    if (st != VMOE_OK) return st;
    trace_before(s, "balance_join");
    st = launch_kernel(balance_join_kernel, dim3(p.T), dim3(FT), 0, s, p, chunks, (const float *)parts, count, tokens,
                       excess, loss);
    trace_after(s);
    return st;
}

int launch_balance_bwd(const Dims &p, const float *logits, const uint8_t *mask, const int32_t *count,
                       const int32_t *tokens, const float *excess, const float *dloss, float *dlogits, cudaStream_t s) {
    trace_before(s, "balance_bwd");
    const int st = with_layout(p.E, [&](auto L, auto V, auto vec) {
        return launch_kernel(balance_bwd_kernel<L(), V(), vec()>, dim3(chunks_of(p), p.T), dim3(BT), 0, s, p, logits,
                             mask, count, tokens, excess, dloss, dlogits);
    });
    trace_after(s);
    return st;
}

}  // namespace vmoe

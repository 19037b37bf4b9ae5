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
// Only tokens that take part are multiplied: head_pack numbers them and copies their rows (fp32 ones as three bf16
// parts), so padding and prompts cost nothing, and what lies in them is not looked at.
//
// Forward: [head_mark] head_pack [head_list] HEAD_STATS or head_few, head_finish; backward: [head_mark] head_pack, then for
// each piece of the vocabulary HEAD_DLOGITS [head_patch] HEAD_DZ HEAD_DW, then [head_dz_join].  17 x 1576 tokens, 32000
// entries, d 768, a head each: 3.4 ms on the same inputs in a row, of it the products 725, 860, 810 and 755 us, packing 28 and 22,
// joining the sums 23; 3.75 on inputs that change, at the power limit.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "head.cuh"

namespace vmoe {
namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr float LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;
constexpr int HG_THREADS = 256, HP_TOKENS = 32, HP_SELF = 2048, HF_DOTS = 16384;
constexpr float PATCH_TAU = 8.0f;
static_assert(HP_TOKENS == 32, "a CTA of head_pack has one word of marks");

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

__device__ __forceinline__ void load8(const float *p, float *o) {
    const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
    o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
}

__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *v) { *reinterpret_cast<uint4 *>(p) = f32_to_bf16x8(v); }
__device__ __forceinline__ void store8(float *p, const float *v) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

struct Sizes {
    int T, N, Np, d, V, K;
};

__device__ __forceinline__ bool entry_ok(const Sizes &z, int i, float l) { return i >= 0 && i < z.V && l != -INFINITY; }
__device__ __forceinline__ bool label_ok(const Sizes &z, int y) { return y >= 0 && y < z.V; }

// Which tokens take part, a bit each: mark [2][T][words], first those with a teacher, then those with either.  A CTA 32
// tokens, four a warp, whose lanes look through a token's entries together.
__global__ void __launch_bounds__(HG_THREADS)
head_mark_kernel(Sizes z, int words, const int32_t *__restrict__ label, const int32_t *__restrict__ tidx,
                 const float *__restrict__ tlogit, unsigned *__restrict__ mark) {
    __shared__ unsigned parts[HG_THREADS / 32];
    const int t = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, word = blockIdx.x, n0 = word * 32;
    pdl_wait();
    pdl_launch_dependents();
    const bool has = warp == 0 && label && n0 + lane < z.N && label_ok(z, label[(long long)t * z.N + n0 + lane]);
    unsigned taught = 0;
    if (tidx) {
        bool some[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = n0 + 4 * warp + i;
            const long long at = ((long long)t * z.N + n) * z.K;
            if (n < z.N)
                for (int j = lane; j < z.K; j += 32) some[i] |= entry_ok(z, tidx[at + j], tlogit[at + j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) taught |= (unsigned)__any_sync(FULL, some[i]) << (4 * warp + i);
    }
    if (lane == 0) parts[warp] = taught;
    const unsigned either = __ballot_sync(FULL, has);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < HG_THREADS / 32; ++i) taught |= parts[i];
        mark[(long long)t * words + word] = taught;
        mark[((long long)z.T + t) * words + word] = either | taught;
    }
}

// Packs the tokens that take part, HP_TOKENS a CTA: how many come before is counted by every CTA, from the bits, or where
// a head has few tokens from their labels and entries themselves.  Copies their rows (fp32 ones as three bf16 parts),
// fills the last block with zeros, and leaves what else belongs to a token: zeros in the outputs of one without a part,
// the backward's factors.
struct Pack {
    Sizes z;
    int words;
    const unsigned *mark;  // NULL: from label, tidx and tlogit
    const int32_t *label, *tidx;
    const float *tlogit;
    int *rows, *pos, *map, *out_label;
    __nv_bfloat16 *out;
    // forward: set to 0 where a token has no part
    float *ce, *lse, *kl, *tlse, *logp;
    // backward
    void *dz;
    bool fill, two;
    float inv_tau;
    bool one;  // labels and a teacher at temperature 1: one exponential for both
    const float *in_ce, *in_lse, *in_tlse, *dce, *dlse, *dkl;
    float4 *coef;
    float *at_label;
};
// At the label dce (p - 1) + dlse p with p = exp(-ce): ce is kept to 2^-24 of itself or of 1, p and 1 would cancel.
__device__ __forceinline__ float label_value(float ce, float dce, float dlse) { return dce * expm1f(-ce) + dlse * expf(-ce); }

template <typename T>
__global__ void __launch_bounds__(HG_THREADS) head_pack_kernel(Pack f, const T *__restrict__ src) {
    __shared__ unsigned bits[2][HP_SELF / 32];  // this head's marks, where they are made here
    __shared__ int sum[2][HG_THREADS / 32], to[HP_TOKENS];
    const Sizes z = f.z;
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n0 = blockIdx.x * HP_TOKENS;
    const long long t0 = (long long)t * z.N;
    if (!f.mark)
        for (int i = tid; i < f.words; i += HG_THREADS) bits[0][i] = bits[1][i] = 0;
    pdl_wait();
    pdl_launch_dependents();
    const unsigned *taught = bits[0], *either = bits[1];
    if (f.mark) {
        taught = f.mark + (long long)t * f.words;
        either = f.mark + ((long long)z.T + t) * f.words;
    } else {
        __syncthreads();
        if (f.tidx) {
#pragma unroll 4
            for (int i = tid; i < z.N * z.K; i += HG_THREADS)
                if (entry_ok(z, f.tidx[t0 * z.K + i], f.tlogit[t0 * z.K + i])) {
                    const int n = i / z.K;
                    atomicOr(bits[0] + (n >> 5), 1u << (n & 31));
                    atomicOr(bits[1] + (n >> 5), 1u << (n & 31));
                }
        }
        __syncthreads();
        if (f.label) {  // a word a warp
#pragma unroll 4
            for (int w = warp; w < f.words; w += HG_THREADS / 32) {
                const int i = w * 32 + lane;
                const unsigned has = __ballot_sync(FULL, i < z.N && label_ok(z, i < z.N ? f.label[t0 + i] : -1));
                if (lane == 0) bits[1][w] |= has;
            }
        }
        __syncthreads();
    }
    int before = 0, total = 0;
    for (int i = tid; i < f.words; i += HG_THREADS) {
        const int c = __popc(either[i]);
        total += c;
        if (i * 32 < n0) before += c;
    }
    before = __reduce_add_sync(FULL, before);
    total = __reduce_add_sync(FULL, total);
    if (lane == 0) sum[0][warp] = before, sum[1][warp] = total;
    __syncthreads();
    before = total = 0;
#pragma unroll
    for (int i = 0; i < HG_THREADS / 32; ++i) before += sum[0][i], total += sum[1][i];
    const int whole = (total + HEAD_HALF - 1) / HEAD_HALF * HEAD_HALF, rows = f.two ? two_row(whole) : total;
    if (blockIdx.x == 0 && tid == 0) f.rows[t] = rows, f.rows[z.T + t] = total;
    const int n = n0 + tid;
    if (tid < HP_TOKENS) to[tid] = -1;
    if (tid < HP_TOKENS && n < z.N) {  // a token a thread
        const unsigned word = either[n >> 5];
        const long long tn = t0 + n;
        const bool in = word >> (n & 31) & 1u;
        int r = before + __popc(word & ((1u << (n & 31)) - 1u));
        if (f.two) r = two_row(r);
        const int y = f.label && label_ok(z, f.label[tn]) ? f.label[tn] : -1;
        f.pos[tn] = to[tid] = in ? r : -1;
        const long long at = (long long)t * z.Np + r;
        if (in) {
            f.map[at] = n;
            if (f.out_label) f.out_label[at] = y;
            if (f.two) {
                f.map[at + HEAD_HALF] = -1;
                if (f.out_label) f.out_label[at + HEAD_HALF] = y;
            }
        } else {
            if (f.ce) f.ce[tn] = f.lse[tn] = 0.0f;
            if (f.kl) f.kl[tn] = f.tlse[tn] = 0.0f;
        }
        if (in && f.coef) {
            // a term that the token does not have: weight 0, and a logarithm that takes its exponential to 0 whatever the logit (from
            // 0 it would be infinite at logits over 88, and 0 times it NaN)
            float4 c = make_float4(0.0f, INFINITY, 0.0f, INFINITY);
            float there = 0.0f;
            if (y >= 0) {
                const float dce = f.dce ? f.dce[tn] : 0.0f, dlse = f.dlse ? f.dlse[tn] : 0.0f;
                there = label_value(f.in_ce[tn], dce, dlse);
                c.x = dce + dlse;
                c.y = f.in_lse[tn] * LOG2E;
            }
            if (f.dkl && (taught[n >> 5] >> (n & 31) & 1u)) {
                const float b = f.dkl[tn] * f.inv_tau;
                if (f.one) {
                    c.x += b;
                    c.y = f.in_tlse[tn] * LOG2E;
                    if (y >= 0) there += b * expf(-f.in_ce[tn]);
                } else {
                    c.z = b;
                    c.w = f.in_tlse[tn] * LOG2E;
                }
            }
            f.coef[at] = c;
            f.at_label[at] = there;
            if (f.two) {
                f.coef[at + HEAD_HALF] = c;
                f.at_label[at + HEAD_HALF] = there;
            }
        }
    }
    __syncthreads();
    // the rows, 8 columns a thread at a time
    const long long plane = (long long)z.T * z.Np * z.d;
    const int vec = z.d / 8, here = min(HP_TOKENS, z.N - n0);
    constexpr int U = sizeof(T) == 2 ? 6 : 3;  // loads in flight a thread
    for (int i0 = tid; i0 < here * vec; i0 += U * HG_THREADS) {
        uint4 v[U][sizeof(T) / 2];
        int r[U], at[U];  // at: token and column
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * HG_THREADS, k = i / vec;
            at[u] = k * z.d + (i - k * vec) * 8;
            r[u] = i < here * vec ? to[k] : -2;
            if (r[u] < 0) continue;
#pragma unroll
            for (int q = 0; q < (int)sizeof(T) / 2; ++q)
                v[u][q] = __ldg(reinterpret_cast<const uint4 *>(src + (t0 + n0) * z.d + at[u]) + q);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r[u] < 0) {
                if (!f.dz || r[u] != -1) continue;
                uint4 *o = reinterpret_cast<uint4 *>((T *)f.dz + (t0 + n0) * z.d + at[u]);
#pragma unroll
                for (int q = 0; q < (int)sizeof(T) / 2; ++q) o[q] = make_uint4(0, 0, 0, 0);
                continue;
            }
            __nv_bfloat16 *o = f.out + ((long long)t * z.Np + r[u]) * z.d + at[u] % z.d;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint4 *>(o) = v[u][0];
                if (f.two) *reinterpret_cast<uint4 *>(o + HEAD_HALF * z.d) = v[u][0];
            } else {
                const float *x = reinterpret_cast<const float *>(v[u]);
                __align__(16) __nv_bfloat16 p[3][8];
#pragma unroll
                for (int q = 0; q < 8; ++q) split3(x[q], p[0][q], p[1][q], p[2][q]);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(o + q * plane) = *reinterpret_cast<const uint4 *>(p[q]);
            }
        }
    }
    if (f.logp)
        for (int i = tid; i < here * z.K; i += HG_THREADS)
            if (to[i / z.K] < 0) f.logp[(t0 + n0) * z.K + i] = 0.0f;
    // the rest of HEAD_DW's last block of tokens, whose sum has zeros times these; elsewhere a row reaches nothing but what is
    // its own, and nobody reads that.  (Whole tiles for everybody: a head of 8 tokens, d 1024, fp32, 30 us a call.)
    if (f.two)  // rows without a token among the first; HEAD_DLOGITS leaves zeros there
        for (int r = 2 * total + blockIdx.x * (HG_THREADS / 32) + warp; r < 2 * whole; r += gridDim.x * (HG_THREADS / 32)) {
            const long long at = (long long)t * z.Np + two_row(r >> 1) + (r & 1) * HEAD_HALF;
            if (lane == 0) f.map[at] = -1;
            for (int c = lane * 8; c < z.d; c += 256) *reinterpret_cast<uint4 *>(f.out + at * z.d + c) = make_uint4(0, 0, 0, 0);
        }
    if (!f.fill) return;
    const int end = (rows + HEAD_BLOCK - 1) / HEAD_BLOCK * HEAD_BLOCK;
    for (int r = rows + blockIdx.x * (HG_THREADS / 32) + warp; r < end; r += gridDim.x * (HG_THREADS / 32)) {
        const long long at = (long long)t * z.Np + r;
        for (int q = 0; q < (sizeof(T) == 2 ? 1 : 3); ++q)
            for (int c = lane * 8; c < z.d; c += 256)
                *reinterpret_cast<uint4 *>(f.out + q * plane + at * z.d + c) = make_uint4(0, 0, 0, 0);
    }
}

// The teacher's entries of 32 packed rows, by the half tile of the vocabulary that they lie in: off [halves + 1] and list
// for the epilogue of HEAD_STATS, which picks their logits.  Order within a half tile does not matter.  A CTA 32 rows.
// 605000 entries: 12 us; a dot product for each took 113, at L2's rate.
__global__ void __launch_bounds__(HG_THREADS)
head_list_kernel(Sizes z, int halves, const int32_t *__restrict__ tidx, const float *__restrict__ tlogit,
                 const int *__restrict__ rows, const int *__restrict__ map, int *__restrict__ off, unsigned *__restrict__ list) {
    extern __shared__ int hl_count[];  // [halves + 1]
    __shared__ int sums[HG_THREADS / 32];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r0 = blockIdx.x * 32;
    pdl_wait();
    pdl_launch_dependents();
    const int n = rows[t];
    if (r0 >= (n + HEAD_TILE - 1) / HEAD_TILE * HEAD_TILE) return;
    const long long block = ((long long)t * z.Np + r0) >> 5;
    for (int i = tid; i <= halves; i += HG_THREADS) hl_count[i] = 0;
    __syncthreads();
    auto each = [&](auto what) {
        for (int i = tid; i < 32 * z.K; i += HG_THREADS) {
            const int r = i / z.K, j = i - r * z.K;
            if (r0 + r >= n) continue;
            const long long at = ((long long)t * z.N + map[(long long)t * z.Np + r0 + r]) * z.K + j;
            const int e = tidx[at];
            if (entry_ok(z, e, tlogit[at])) what(r, j, e);
        }
    };
    each([&](int, int, int e) { atomicAdd(hl_count + (e >> 7), 1); });
    __syncthreads();
    // exclusive sums, a run of half tiles a thread
    const int per = (halves + 1 + HG_THREADS - 1) / HG_THREADS, i0 = min(halves + 1, tid * per), i1 = min(halves + 1, i0 + per);
    int mine = 0;
    for (int i = i0; i < i1; ++i) mine += hl_count[i];
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(FULL, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    int run = incl - mine;
    for (int i = 0; i < warp; ++i) run += sums[i];
    for (int i = i0; i < i1; ++i) {
        const int c = hl_count[i];
        hl_count[i] = run;
        off[block * (halves + 1) + i] = run;
        run += c;
    }
    __syncthreads();
    unsigned *out = list + block * 32 * z.K;
    each([&](int r, int j, int e) {
        out[atomicAdd(hl_count + (e >> 7), 1)] = (unsigned)r | (unsigned)(e & 127) << 5 | (unsigned)j << 12;
    });
}

// fp32 weights as three bf16 parts.  n: a multiple of 8.
__global__ void __launch_bounds__(HG_THREADS)
head_split_kernel(long long n, const float *__restrict__ src, __nv_bfloat16 *__restrict__ out) {
    pdl_wait();
    pdl_launch_dependents();
    for (long long i = ((long long)blockIdx.x * HG_THREADS + threadIdx.x) * 8; i < n; i += (long long)gridDim.x * HG_THREADS * 8) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(src + i)), b = __ldg(reinterpret_cast<const float4 *>(src + i) + 1);
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint4 p[3];
        split_weights(v, p);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4 *>(out + q * n + i) = p[q];
    }
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

// The losses from the tiles' sums, ROWS packed rows a CTA: 256 / ROWS threads join a row's half tiles, every one of them
// a share, then their sums; with a teacher a warp then takes a row's entries.
struct Finish {
    Sizes z;
    int halves, pitch;  // half tiles of the vocabulary, and as the sums are laid out
    int stats;
    float inv_tau, c1, c2;  // c2: of the teacher's sum
    const int *rows, *map, *label;
    const float2 *part, *part2;
    const float *picked, *tl;
    const void *dot_z, *dot_w;  // few entries: their logits are formed here, from the tokens and weights
    const int32_t *tidx;
    const float *tlogit;
    float *ce, *lse, *kl, *tlse, *logp;
};
__device__ __forceinline__ void join(float &m, float &s, float2 v) {
    const float top = fmaxf(m, v.x);
    s = s * exp2f(m - top) + v.y * exp2f(v.x - top);
    m = top;
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *o) { bf16x8_to_f32(__ldg(reinterpret_cast<const uint4 *>(p)), o); }

// Lane l < 8: the logit of entry i of lane l; all eight rows at a time.
template <typename T>
__device__ __forceinline__ float entries_logits(int d, const T *zr, const T *w, int i) {
    constexpr int U = 8;
    const int lane = threadIdx.x & 31;
    float acc[U] = {}, mine = 0.0f;
    const T *row[U];
#pragma unroll
    for (int e = 0; e < U; ++e) row[e] = w + (long long)max(0, __shfl_sync(FULL, i, e)) * d;
#pragma unroll 2
    for (int c = lane * 8; c < d; c += 256) {
        float a[8], b[U][8];
        load8(zr + c, a);
#pragma unroll
        for (int e = 0; e < U; ++e) load8(row[e] + c, b[e]);
#pragma unroll
        for (int e = 0; e < U; ++e)
#pragma unroll
            for (int x = 0; x < 8; ++x) acc[e] = fmaf(a[x], b[e][x], acc[e]);
    }
#pragma unroll
    for (int e = 0; e < U; ++e) {
        acc[e] = warp_sum(acc[e]);
        if (lane == e) mine = acc[e];
    }
    return mine;
}

// DOTS: void, or the type of z and w where the entries' logits are formed here.
template <int ROWS, typename DOTS>
__global__ void __launch_bounds__(HG_THREADS) head_finish_kernel(Finish f) {
    constexpr int SHARES = HG_THREADS / ROWS;  // threads of a row
    __shared__ float2 sm[2][HG_THREADS / 32][ROWS];
    __shared__ float tl[ROWS];
    __shared__ float2 top[ROWS];  // the teacher's sum, in units of log2: largest logit, logarithm
    constexpr bool DOT = !std::is_void<DOTS>::value;
    __shared__ float dots[DOT ? ROWS : 1][DOT ? HEAD_K : 1];
    const int t = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row_in = lane % ROWS;
    const Sizes z = f.z;
    pdl_wait();
    pdl_launch_dependents();
    const int n = f.rows[t], r0 = blockIdx.x * ROWS;
    if (r0 >= n) return;
    const int row = r0 + row_in;
    float m = -3e38f, s = 0.0f, m2 = -3e38f, s2 = 0.0f;
    const float2 *p = f.part + (long long)t * f.pitch * z.Np + row;
    const float2 *p2 = f.stats == 2 ? f.part2 + (long long)t * f.pitch * z.Np + row : nullptr;
#pragma unroll 4
    for (int h = tid / ROWS; h < f.halves; h += SHARES) {
        join(m, s, p[(long long)h * z.Np]);
        if (p2) join(m2, s2, p2[(long long)h * z.Np]);
    }
#pragma unroll
    for (int o = 16; o >= ROWS; o >>= 1) {
        join(m, s, make_float2(__shfl_xor_sync(FULL, m, o), __shfl_xor_sync(FULL, s, o)));
        join(m2, s2, make_float2(__shfl_xor_sync(FULL, m2, o), __shfl_xor_sync(FULL, s2, o)));
    }
    if (lane < ROWS) {
        sm[0][warp][lane] = make_float2(m, s);
        sm[1][warp][lane] = make_float2(m2, s2);
    }
    __syncthreads();
    if (tid < ROWS) {
        for (int q = 1; q < HG_THREADS / 32; ++q) {
            join(m, s, sm[0][q][lane]);
            join(m2, s2, sm[1][q][lane]);
        }
        const float ls = log2f(s), a = (m + ls) * LN2;
        top[lane] = p2 ? make_float2(m2, log2f(s2)) : make_float2(m, ls);
        tl[lane] = (top[lane].x + top[lane].y) * LN2;
        if (row < n && f.ce) {
            const long long at = (long long)t * z.Np + row, tn = (long long)t * z.N + f.map[at];
            const bool has = f.label[at] >= 0;
            f.ce[tn] = has ? ((m - f.picked[at] * f.c1) + ls) * LN2 : 0.0f;  // a sure token's is small: no difference of large ones
            f.lse[tn] = has ? a : 0.0f;
        }
    }
    if (!f.kl) return;
    if constexpr (DOT) {  // eight entries of a row a warp
        const int each = (z.K + 7) / 8;
        for (int b = warp; b < min(ROWS, n - r0) * each; b += HG_THREADS / 32) {
            const int i = b / each, j = (b - i * each) * 8 + lane;
            const long long tn = (long long)t * z.N + f.map[(long long)t * z.Np + r0 + i];
            int e = -1;
            if (lane < 8 && j < z.K) {
                e = f.tidx[tn * z.K + j];
                if (!entry_ok(z, e, f.tlogit[tn * z.K + j])) e = -1;
            }
            const float l = entries_logits(z.d, (const DOTS *)f.dot_z + tn * z.d, (const DOTS *)f.dot_w + (long long)t * z.V * z.d, e);
            if (e >= 0) dots[i][j] = l;
        }
    }
    __syncthreads();
    for (int i = warp; i < ROWS && r0 + i < n; i += HG_THREADS / 32) {
        const long long at = (long long)t * z.Np + r0 + i, tn = (long long)t * z.N + f.map[at];
        Teacher q;
        q.load(z, f.tidx, f.tlogit, f.inv_tau, tn);
        float loss = 0.0f;
#pragma unroll
        for (int mm = 0; mm < Teacher::M; ++mm) {
            if (32 * mm >= z.K) break;
            const int j = lane + 32 * mm;
            float l = 0.0f;
            if (j < z.K && q.i[mm] >= 0) l = DOT ? dots[DOT ? i : 0][DOT ? j : 0] : f.tl[at * z.K + j];
            if (j >= z.K) continue;
            // not l / tau - tlse, whose difference of large numbers is off by 2e-6 where a sure teacher and a sure model leave p - q
            const float lp = q.i[mm] >= 0 ? (fmaf(l, f.c2, -top[i].x) - top[i].y) * LN2 : 0.0f;
            f.logp[tn * z.K + j] = lp;
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

// The teacher's entries in a piece of dl: the whole value, from the stored logarithms, so that neither the order of
// equal entries nor a label among them matters.  A warp a packed row.  605000 entries of the six-task step: 28 us, single
// values written into rows that L2 no longer holds.
// The other softmax at an entry, exp(l - lse), has l from tau (logp + tlse), whose roundings tau multiplies: p is off by
// tau 2^-24 (|logp| + |tlse|) of itself: 1e-5 at PATCH_TAU, all of it at 10^6.  Above PATCH_TAU l is formed again as a dot product
// (DOTS: the type of z and w, else void), which reads a row of w an entry: the six-task step's backward 900 -> 1023 us.
struct Patch {
    Sizes z;
    int v0, vn, piece, parts;
    float tau, inv_tau;
    const int *rows, *map;
    const int32_t *label, *tidx;
    const float *tlogit, *ce, *lse, *tlse, *logp, *dce, *dlse, *dkl;
    const void *dot_z, *dot_w;
    __nv_bfloat16 *dl;
};
template <typename DOTS>
__global__ void __launch_bounds__(HG_THREADS) head_patch_kernel(Patch f) {
    constexpr bool DOT = !std::is_void<DOTS>::value;
    const int t = blockIdx.y, lane = threadIdx.x & 31, r = blockIdx.x * (HG_THREADS / 32) + (threadIdx.x >> 5);
    const Sizes z = f.z;
    pdl_wait();
    pdl_launch_dependents();
    if (r >= f.rows[t]) return;
    const long long at = (long long)t * z.Np + r, tn = (long long)t * z.N + f.map[at];
    if (f.map[at] < 0) return;
    Teacher q;
    q.load(z, f.tidx, f.tlogit, f.inv_tau, tn);
    if (!q.any) return;
    const int y = f.label && label_ok(z, f.label[tn]) ? f.label[tn] : -1;
    const float dce = y >= 0 && f.dce ? f.dce[tn] : 0.0f, dlse = y >= 0 && f.dlse ? f.dlse[tn] : 0.0f;
    const float b = f.dkl[tn] * f.inv_tau, lse = y >= 0 ? f.lse[tn] : 0.0f, tlse = f.tlse[tn];
    const long long plane = (f.parts == 2 ? HEAD_HALF : (long long)z.T * z.Np) * f.piece;
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
        const bool here = i >= f.v0 && i < f.v0 + f.vn;
        float l = 0.0f;
        if constexpr (DOT) {  // eight entries at a time
            if (y >= 0)
                for (int j = 0; j < 4; ++j) {
                    if (!__any_sync(FULL, here && lane / 8 == j)) continue;
                    const float each = entries_logits(z.d, (const DOTS *)f.dot_z + tn * z.d, (const DOTS *)f.dot_w + (long long)t * z.V * z.d,
                                                      __shfl_sync(FULL, i, 8 * j + (lane & 7)));
                    const float mine = __shfl_sync(FULL, each, lane & 7);
                    if (lane / 8 == j) l = mine;
                }
        }
        if (!here) continue;
        const float lp = f.logp[tn * z.K + lane + 32 * m];
        float v = b * (expf(lp) - all);
        if (y >= 0) v += i == y ? label_value(f.ce[tn], dce, dlse) : (dce + dlse) * expf((DOT ? l : f.tau * (lp + tlse)) - lse);
        __nv_bfloat16 *o = row + (i - f.v0);
        if (f.parts < 3) {
            const __nv_bfloat16 hi = __float2bfloat16_rn(v);
            o[0] = hi;
            if (f.parts == 2) o[plane] = __float2bfloat16_rn(v - __bfloat162float(hi));
        } else {
            split3(v, o[0], o[plane], o[2 * plane]);
        }
    }
}

// dz from its sums over the pieces of the vocabulary; 0 for a token without a part.  Eight columns a thread.
template <typename T>
__global__ void __launch_bounds__(HG_THREADS)
head_dz_kernel(Sizes z, const int *__restrict__ pos, const float *__restrict__ sums, T *__restrict__ dz) {
    pdl_wait();
    pdl_launch_dependents();
    const int vec = z.d / 8;
    const long long total = (long long)z.T * z.N * vec;
    for (long long i = (long long)blockIdx.x * HG_THREADS + threadIdx.x; i < total; i += (long long)gridDim.x * HG_THREADS) {
        const long long tn = i / vec;
        const int c = (int)(i - tn * vec) * 8, r = pos[tn];
        float v[8] = {};
        if (r >= 0) load8(sums + ((tn / z.N) * z.Np + r) * z.d + c, v);
        store8(dz + tn * z.d + c, v);
    }
}

// The tiles of dz whose sums were cut (DzShares), from their parts in order.  A CTA eight rows of a tile.
template <typename T>
__global__ void __launch_bounds__(HG_THREADS)
head_dz_join_kernel(Sizes z, int pairs, int kb, int least, int tiles_n, const int *__restrict__ rows, const int *__restrict__ map,
                    const float *__restrict__ parts, T *__restrict__ dz) {
    pdl_wait();
    pdl_launch_dependents();
    int tiles = 0;
    for (int t = 0; t < z.T; ++t) tiles += (rows[t] + HEAD_TILE - 1) / HEAD_TILE * tiles_n;
    const DzShares s(tiles, pairs, kb, least);
    const int tile = blockIdx.x;
    if (tile >= s.left || s.cuts == 1) return;
    int local = s.full + tile, t = 0, n = 0;
    for (;; ++t) {
        n = rows[t];
        const int c = (n + HEAD_TILE - 1) / HEAD_TILE * tiles_n;
        if (local < c) break;
        local -= c;
    }
    const int in = blockIdx.y * 8 + (threadIdx.x >> 5), r = local / tiles_n * HEAD_TILE + in;
    const int c0 = (threadIdx.x & 31) * 8, col = local % tiles_n * HEAD_TILE + c0;
    if (r >= n || col >= z.d || map[(long long)t * z.Np + r] < 0) return;
    T *o = dz + ((long long)t * z.N + map[(long long)t * z.Np + r]) * z.d + col;
    const float *p = parts + ((long long)tile * HEAD_TILE + in) * HEAD_TILE + c0;
    const long long step = (long long)s.left * HEAD_TILE * HEAD_TILE;
    float v[8] = {};
    constexpr int U = 8;  // parts in flight
    for (int cut = 0; cut < s.cuts; cut += U) {
        float b[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) load8(p + min(cut + u, s.cuts - 1) * step, b[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (cut + u < s.cuts)
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] += b[u][q];
    }
    store8(o, v);
}

Sizes sizes_of(const HeadPlan &h) { return Sizes{h.T, h.N, h.Np, h.d, h.V, h.K}; }
template <typename P>
P *at(void *ws, size_t offset) {
    return reinterpret_cast<P *>(static_cast<uint8_t *>(ws) + offset);
}

// Packed rows and, in fp32, the weights' parts: what both directions begin with.  f: what the direction adds.
int prepare(const Dims &p, const HeadPlan &h, const HeadIn &in, void *ws, Pack f, const __nv_bfloat16 **zp,
            const __nv_bfloat16 **wp, bool split, cudaStream_t s) {
    const Sizes z = sizes_of(h);
    f.z = z;
    f.words = (h.N + 31) / 32;
    f.label = in.label;
    f.rows = at<int>(ws, h.rows);
    f.pos = at<int>(ws, h.pos);
    f.map = at<int>(ws, h.map);
    f.out_label = in.label ? at<int>(ws, h.label) : nullptr;
    f.out = at<__nv_bfloat16>(ws, h.z);
    int st;
    f.tidx = in.tidx;
    f.tlogit = in.tlogit;
    // few labels and entries: every CTA of head_pack looks through all of its head's, instead of a launch (8192 tokens: 24 us
    // so, 21 with the marks)
    if (h.N > HP_SELF || (in.tidx && (long long)h.N * h.K > HF_DOTS)) {
        unsigned *mark = at<unsigned>(ws, h.mark);
        f.mark = mark;
        trace_before(s, "head_mark");
        st = launch_kernel(head_mark_kernel, dim3(f.words, h.T), dim3(HG_THREADS), 0, s, z, f.words, in.label, in.tidx, in.tlogit, mark);
        trace_after(s);
        if (st != VMOE_OK) return st;
    }
    trace_before(s, "head_pack");
    const dim3 grid((h.N + HP_TOKENS - 1) / HP_TOKENS, h.T);
    st = p.bf16 ? launch_kernel(head_pack_kernel<__nv_bfloat16>, grid, dim3(HG_THREADS), 0, s, f, (const __nv_bfloat16 *)in.z)
                : launch_kernel(head_pack_kernel<float>, grid, dim3(HG_THREADS), 0, s, f, (const float *)in.z);
    trace_after(s);
    if (st != VMOE_OK) return st;
    *zp = f.out;
    *wp = (const __nv_bfloat16 *)in.w;
    if (split) {
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
    // dl is an operand of the tensor cores and in bf16 problems a bf16 value, off by up to 2^-8, 1.6e-3 in the mean, which sums
    // of independent roundings keep: dz and dw are 2.3e-3 off where their own rounding alone is 1.66e-3.  Two rows a token keep it to
    // 2^-16 and take twice the products.  That costs nothing up to 128 tokens, which leave half of a tile's rows empty, and little
    // while the logits' tiles, doubled, are still one a pair (forward and backward, one row a token and two, us: 197 tokens, 1000 entries
    // 72 and 71, 9000 77 and 84); beyond, it is a choice for the time that bf16 training makes (197 x 128000 236 and 298; 1024 x 40000
    // 212 and 311; 1024 x 128000 520 and 841).
    const size_t rows2 = ((size_t)two_row((h.N + HEAD_HALF - 1) / HEAD_HALF * HEAD_HALF) + HEAD_TILE - 1) / HEAD_TILE * HEAD_TILE;
    h.two = p.bf16 && h.N <= HEAD_TILE &&
            (h.N <= HEAD_TILE / 2 || (size_t)h.T * (rows2 / HEAD_TILE) * ((h.V + HEAD_TILE - 1) / HEAD_TILE) <= (size_t)num_sms() / 2);
    if (h.two) h.Np = (int)rows2;
    // a warp 32 (fp32: 16) entries at a time, two CTAs of eight warps an SM.  4 tokens, us so and as tiles: 128000 entries in bf16, d 2048
    // 110 and 116, 2560 137 and 137, 4096, where an SM holds the tokens once, 218 and 199; 50000 in fp32, d 1024 98 and 212; wider ones
    // (1536, held once: 116 and 309) are still tiles
    if (h.N <= HEAD_FEW && h.d <= (p.bf16 ? 2048 : 1024))
        h.few = std::max(1, std::min((h.V + 255) / 256, std::max(1, 2 * num_sms() / h.T)));
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
    h.rows = take((size_t)h.T * 8);
    h.mark = take((size_t)h.T * ((h.N + 31) / 32) * 8);
    h.pos = take((size_t)h.T * h.N * 4);
    h.map = take(rowsp * 4);
    h.label = take(rowsp * 4);
    h.z = take(rowsp * h.d * 2 * h.parts);
    h.w = take(p.bf16 ? 0 : (size_t)h.T * h.V * h.d * 6);
    const size_t both = o;
    h.part = take(rowsp * tiles_v * 2 * 8);
    h.part2 = take(h.K > 0 ? rowsp * tiles_v * 2 * 8 : 0);
    h.picked = take(rowsp * 4);
    h.off = take(h.K > 0 ? rowsp / 32 * (tiles_v * 2 + 1) * 4 : 0);
    h.list = take(rowsp * h.K * 4);
    h.tl = take(rowsp * h.K * 4);
    const size_t fwd = o;
    o = both;
    h.coef = take(rowsp * 16);
    h.at_label = take(rowsp * 4);
    const size_t fixed = o, column = rowsp * HEAD_TILE * 2 * h.parts;  // a tile of columns of dl
    // the whole vocabulary at once where there is room: dz is then shared out to the SM pairs.  Backward in pieces and at once, us,
    // d 1024: 16384 tokens, 128000 entries 7990 and 7870; 2304 tokens, 500000 entries, whose tiles of dz leave pairs idle, 4980 and 4170
    const size_t tiles_d = rowsp / HEAD_TILE * ((h.d + HEAD_TILE - 1) / HEAD_TILE), blocks = ((size_t)h.V + 63) / 64;
    const size_t pairs = std::min<size_t>(std::max(1, num_sms() / 2), std::max(tiles_d, tiles_d * blocks / dz_least(h.parts)));
    const size_t whole = pairs * HEAD_TILE * HEAD_TILE * 4, sums = (rowsp * h.d * 4 + 255) & ~(size_t)255;
    if (bytes && bytes < fwd) return false;
    size_t cols = tiles_v;
    const size_t have = bytes ? bytes : fixed + std::max(whole, sums) + std::max(column, (size_t)2 << 30);
    if (have >= fixed + whole + tiles_v * column) {
        h.pairs = (int)pairs;
    } else {
        if (have < fixed + sums + column) return false;
        cols = std::min(tiles_v, (have - fixed - sums) / column);
    }
    h.piece = (int)(cols * HEAD_TILE);
    h.dl = take(cols * column);
    h.dzp = take(h.pairs ? whole : sums);
    h.bytes = std::max(o, fwd);
    *out = h;
    return true;
}

size_t head_min_workspace(const Dims &p, const vmoe_head *head) {
    HeadPlan h;
    if (!head_plan(p, head, true, 0, &h)) return 0;
    const size_t rowsp = (size_t)h.T * h.Np, dzp = (rowsp * h.d * 4 + 255) & ~(size_t)255;
    const size_t bwd = h.dl + rowsp * HEAD_TILE * 2 * h.parts + dzp;
    return std::max(h.tl + ((rowsp * h.K * 4 + 255) & ~(size_t)255), bwd);
}

int launch_head_loss(const Dims &p, const HeadPlan &h, const HeadIn &in, float *ce, float *lse, float *kl, float *tlse,
                     float *logp, void *ws, cudaStream_t s) {
    const __nv_bfloat16 *zp, *wp;
    Pack k = {};
    k.ce = ce;
    k.lse = lse;
    k.kl = kl;
    k.tlse = tlse;
    k.logp = logp;
    int st = prepare(p, h, in, ws, k, &zp, &wp, !p.bf16 && !h.few, s);
    if (st != VMOE_OK) return st;
    const Sizes z = sizes_of(h);
    const int pitch = (h.V + HEAD_TILE - 1) / HEAD_TILE * 2;
    HeadGemm g = {};
    g.rows = at<int>(ws, h.rows);
    g.vn = h.V;
    // few entries: a dot product each in head_finish, instead of a launch for their list
    const bool dots = in.tidx && (h.few || (long long)h.T * h.N * h.K <= HF_DOTS);
    if (in.tidx && !dots) {
        int *off = at<int>(ws, h.off);
        unsigned *list = at<unsigned>(ws, h.list);
        g.off = off;
        g.list = list;
        g.K = h.K;
        g.tl = at<float>(ws, h.tl);
        trace_before(s, "head_list");
        st = launch_kernel(head_list_kernel, dim3(h.Np / 32, h.T), dim3(HG_THREADS), (size_t)(pitch + 1) * 4, s, z, pitch, in.tidx,
                           in.tlogit, g.rows, at<int>(ws, h.map), off, list);
        trace_after(s);
        if (st != VMOE_OK) return st;
    }
    g.label = in.label ? at<int>(ws, h.label) : nullptr;
    g.part = at<float2>(ws, h.part);
    g.part2 = at<float2>(ws, h.part2);
    g.picked = at<float>(ws, h.picked);
    st = h.few ? launch_head_few(h, g, zp, in.w, s) : launch_head_gemm(HEAD_STATS, h, g, zp, wp, nullptr, nullptr, s);
    if (st != VMOE_OK) return st;
    Finish f = {};
    f.z = z;
    f.halves = h.few ? h.few : (h.V + 127) / 128;
    f.pitch = h.few ? h.few : pitch;
    f.stats = h.stats;
    f.inv_tau = 1.0f / h.tau;
    f.c1 = h.c1;
    f.c2 = h.stats == 2 ? h.c2 : h.c1;
    f.rows = g.rows;
    f.map = at<int>(ws, h.map);
    f.label = at<int>(ws, h.label);
    f.part = g.part;
    f.part2 = g.part2;
    f.picked = g.picked;
    f.tl = g.tl;
    f.dot_z = in.z;
    f.dot_w = in.w;
    f.tidx = in.tidx;
    f.tlogit = in.tlogit;
    f.ce = ce;
    f.lse = lse;
    f.kl = kl;
    f.tlse = tlse;
    f.logp = logp;
    trace_before(s, "head_finish");
    // few rows: more threads each, to hide the chain of their half tiles
    const bool few = (long long)h.T * h.N <= 2048;
    const int rows = !few ? 32 : dots && h.K > 32 ? 1 : 4;  // a row's entries keep its warps busy
    auto kern = !dots    ? (few ? head_finish_kernel<4, void> : head_finish_kernel<32, void>)
                : p.bf16 ? (rows == 1   ? head_finish_kernel<1, __nv_bfloat16>
                            : rows == 4 ? head_finish_kernel<4, __nv_bfloat16>
                                        : head_finish_kernel<32, __nv_bfloat16>)
                         : (rows == 1   ? head_finish_kernel<1, float>
                            : rows == 4 ? head_finish_kernel<4, float>
                                        : head_finish_kernel<32, float>);
    st = launch_kernel(kern, dim3((h.N + rows - 1) / rows, h.T), dim3(HG_THREADS), 0, s, f);
    trace_after(s);
    return st;
}

int launch_head_loss_bwd(const Dims &p, const HeadPlan &h, const HeadIn &in, const float *ce, const float *lse,
                         const float *tlse, const float *logp, const float *dce, const float *dlse, const float *dkl, void *dz,
                         void *dw, void *ws, cudaStream_t s) {
    const __nv_bfloat16 *zp, *wp;
    Pack k = {};
    k.dz = dz;
    k.fill = dw != nullptr;
    k.two = h.two;
    k.inv_tau = 1.0f / h.tau;
    k.one = h.stats == 1;
    k.in_ce = ce;
    k.in_lse = lse;
    k.in_tlse = tlse;
    k.dce = dce;
    k.dlse = dlse;
    k.dkl = dkl;
    k.coef = at<float4>(ws, h.coef);
    k.at_label = at<float>(ws, h.at_label);
    int st = prepare(p, h, in, ws, k, &zp, &wp, !p.bf16, s);
    if (st != VMOE_OK) return st;
    const Sizes z = sizes_of(h);
    const int *rows = at<int>(ws, h.rows), *map = at<int>(ws, h.map);
    const bool direct = h.pairs > 0;  // dz in one go
    const int pairs = direct && dz ? std::min(h.pairs, head_dz_pairs(h.parts)) : 0;
    if (direct && dz && pairs == 0) return VMOE_ERR_CUDA;
    __nv_bfloat16 *dl = at<__nv_bfloat16>(ws, h.dl);
    HeadGemm g = {};
    g.rows = rows;
    g.label = in.label ? at<int>(ws, h.label) : nullptr;
    g.coef = k.coef;
    g.at_label = k.at_label;
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
            f.parts = h.two ? 2 : h.parts;
            f.tau = h.tau;
            f.inv_tau = k.inv_tau;
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
            f.dot_z = in.z;
            f.dot_w = in.w;
            auto kern = !(in.label && h.tau > PATCH_TAU) ? head_patch_kernel<void>
                        : p.bf16                         ? head_patch_kernel<__nv_bfloat16>
                                                         : head_patch_kernel<float>;
            trace_before(s, "head_patch");
            st = launch_kernel(kern, dim3(((h.two ? two_row(h.N - 1) + 1 : h.N) + 7) / 8, h.T), dim3(HG_THREADS), 0, s, f);
            trace_after(s);
            if (st != VMOE_OK) return st;
        }
        if (dz) {
            g.out = at<float>(ws, h.dzp);
            g.dz = direct ? dz : nullptr;
            g.pairs = pairs;
            g.map = map;
            g.N = h.N;
            g.overlap = dw != nullptr && pdl_enabled();
            if ((st = launch_head_gemm(HEAD_DZ, h, g, zp, wp, dl, nullptr, s)) != VMOE_OK) return st;
            g.pairs = 0;
        }
        if (dw) {
            g.out = (float *)dw;
            g.overlap = dz != nullptr && pdl_enabled();
            if ((st = launch_head_gemm(HEAD_DW, h, g, zp, wp, dl, (__nv_bfloat16 *)dw, s)) != VMOE_OK) return st;
        }
    }
    if (!dz || (direct && (h.V + 63) / 64 < 2 * dz_least(h.parts))) return VMOE_OK;  // no tile was cut
    trace_before(s, "head_dz_join");
    const int *pos = at<int>(ws, h.pos);
    const float *parts = at<float>(ws, h.dzp);
    if (direct) {
        const int kb = (h.V + 63) / 64, least = dz_least(h.parts), tiles_n = (h.d + HEAD_TILE - 1) / HEAD_TILE;
        const dim3 grid(pairs, HEAD_TILE / 8);
        st = p.bf16 ? launch_kernel(head_dz_join_kernel<__nv_bfloat16>, grid, dim3(HG_THREADS), 0, s, z, pairs, kb, least, tiles_n, rows,
                                    map, parts, (__nv_bfloat16 *)dz)
                    : launch_kernel(head_dz_join_kernel<float>, grid, dim3(HG_THREADS), 0, s, z, pairs, kb, least, tiles_n, rows, map,
                                    parts, (float *)dz);
    } else {
        const long long blocks = ((long long)h.T * h.N * (h.d / 8) + HG_THREADS - 1) / HG_THREADS;
        const dim3 grid((unsigned)std::min(blocks, 16LL * num_sms()));
        st = p.bf16 ? launch_kernel(head_dz_kernel<__nv_bfloat16>, grid, dim3(HG_THREADS), 0, s, z, pos, parts, (__nv_bfloat16 *)dz)
                    : launch_kernel(head_dz_kernel<float>, grid, dim3(HG_THREADS), 0, s, z, pos, parts, (float *)dz);
    }
    trace_after(s);
    return st;
}

}  // namespace vmoe
